"""GPU tests of what shares a pool of pages with what: padded prompts take the pages of their own lengths, sequences whose
prompts found none emit nothing, whatever becomes free later."""
import pytest
import torch

from paper_2609_21704_amd import _lib
from paper_2609_21704_amd import decoder as dec
from paper_2609_21704_amd import synth
from paper_2609_21704_amd.engine import Engine
from test_gpu_engine import check_greedy, parent_model, ragged_prompts
from test_gpu_paged_decoder import config, padded

pytestmark = pytest.mark.gpu
DEV = "cuda"


# ------------------------------------------------------------ padded prompts
@pytest.mark.parametrize("route", ["f16", "int4", "fp8"])
@pytest.mark.parametrize("lengths,pages", [([10, 200], 6), ([200, 10], 6), ([130, 5], 4), ([64, 65, 193], 8)])
def test_padded_prompts_take_their_own_pages(route, lengths, pages):
    """A pool that holds the prompts but not their padding, with pages that other prompts have written before."""
    cfg, max_new = config(len(lengths)), 12
    eng = Engine(cfg, DEV, layers=3, k=3, batch=len(lengths), capacity=256, temperature=0.0, pages=pages)
    d = eng.decoder(route)
    for cache in (d.pcache, d.dcache):
        for a in cache.arrays if cache else ():
            a.copy_(torch.randn(a.shape, device=DEV).to(a.dtype))
    prompts = ragged_prompts(cfg, lengths, 21)
    got = [r.tokens for r in eng.generate(prompts, max_new, routes=[route] * len(prompts))]
    dims, model = parent_model(eng.weights["f16"])
    for i, p in enumerate(prompts):
        assert len(got[i]) == max_new
        check_greedy(dims, model, p, got[i], f"{route} {i}")


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("route", ["f16", "int4"])
def test_prompts_that_do_not_fit_end_their_batch(route, packed):
    """... before any of its rounds; the next batch is served."""
    cfg = config(3)
    eng = Engine(cfg, DEV, layers=3, k=3, batch=3, capacity=256, temperature=0.0, pages=5, packed=packed)
    long, short = ragged_prompts(cfg, [130, 140, 60], 22), ragged_prompts(cfg, [30, 66, 20], 23)
    with pytest.raises(RuntimeError, match="pages .*status flags"):
        eng.generate(long, 9, routes=[route] * 3)
    assert eng.stats()["rounds"][route] == 0
    got = [r.tokens for r in eng.generate(short, 9, routes=[route] * 3)]
    dims, model = parent_model(eng.weights["f16"])
    for i, p in enumerate(short):
        check_greedy(dims, model, p, got[i], f"{route} {i}")


@pytest.mark.parametrize("how", ["padded", "packed", "samples"])
def test_a_prompt_without_pages_never_speaks(how):
    """Pages that become free later hold nothing of it: its sequence stays silent, the others go on."""
    samples = 2 if how == "samples" else 1
    cfg = config(4 if samples == 2 else 3)
    w = dec.DecoderWeights(cfg, DEV)
    lengths = [70, 140] if samples == 2 else [70, 140, 40]
    prompts = ragged_prompts(cfg, lengths, 24)
    # 70 and 140 positions take 2 and 3 pages, their samples one more each
    d = dec.DirectDecoder(w, capacity=256, temperature=0.0, pages=5 if samples == 2 else 4, samples=samples)
    for a in d.pcache.arrays:
        a.copy_(torch.randn(a.shape, device=DEV).to(a.dtype))
    if how == "padded":
        d.prefill(padded(prompts), lengths=lengths)
    else:
        d.prefill_packed(prompts)
    assert d.status.item() & _lib.DEV_NO_PAGES
    for r in range(8):
        if r == 4:  # the first sequence ends, and its pages are free
            keep = torch.tensor([0] + [-1] * (cfg.batch - 1), dtype=torch.int32, device=DEV)
            d.pages.trim(keep)
            d.pos_base.masked_fill_(keep == 0, -1)
        d.run()
    # of the rows with pages: the first prompt's for 4 rounds, until it ends; the second one's where samples have none
    want = [4, 0, 8, 0] if samples == 2 else [4, 0, 0]
    assert d.out_len.tolist() == want
    dims, model = parent_model(w)
    for s, n in enumerate(want):
        if n:
            check_greedy(dims, model, prompts[s // samples], d.out_tokens[s, :n].tolist(), f"row {s}")


@pytest.mark.parametrize("chunk", [None, 9])
def test_padding_past_the_pages_raises_no_status(chunk):
    """Padding has no pages past its prompt's own; what it meets there is no fault, another fault still is."""
    cfg = config(2)
    w = dec.DecoderWeights(cfg, DEV)
    prompts = ragged_prompts(cfg, [10, 200], 25)
    d = dec.SpecDecoder(w, capacity=256, temperature=0.0, pages=6)
    d.prefill(padded(prompts), lengths=[10, 200], chunk=chunk)
    assert d.status.item() == 0 and d.pages.held.tolist() == [1, 4]
    for _ in range(4):
        d.run()
    assert d.status.item() == 0
    dims, model = parent_model(w)
    for i, p in enumerate(prompts):
        check_greedy(dims, model, p, d.out_tokens[i, :int(d.out_len[i])].tolist(), f"sequence {i}")
    tokens = padded(prompts)
    tokens[1, 7] = cfg.vocab
    d.prefill(tokens, lengths=[10, 200], chunk=chunk)
    assert d.status.item() == _lib.DEV_BAD_TOKEN
