"""GPU tests of the decoders and the engine over paged caches and with sampling filters: the parent's greedy tokens, samples
that share their prompt's pages, pools that run out, compaction between steps, rounds that emit filtered tokens only."""
import pytest
import torch

from paper_2609_21704_amd import _lib
from paper_2609_21704_amd import decoder as dec
from paper_2609_21704_amd import synth
from paper_2609_21704_amd.configs import Config
from paper_2609_21704_amd.engine import Engine
from test_gpu_engine import agree_until_near_tie, check_greedy, parent_model, ragged_prompts

pytestmark = pytest.mark.gpu
DEV = "cuda"


def config(batch=3, variant="int4"):
    return Config(0, "paged", 3, 512, 1152, 4, 2, 1000, variant, 3, batch, 5)


def padded(prompts):
    t = torch.zeros((len(prompts), max(map(len, prompts))), dtype=torch.int32)
    for i, p in enumerate(prompts):
        t[i, :len(p)] = torch.tensor(p, dtype=torch.int32)
    return t


@pytest.mark.parametrize("packed,draft_cache", [(False, "f16"), (True, "f16"), (True, "q4")])
def test_engine_over_pages(packed, draft_cache):
    """Every route emits the parent's greedy tokens, as over contiguous caches."""
    cfg, lengths, max_new = config(2), [70, 5, 128, 63], 14
    args = dict(layers=3, k=3, batch=2, capacity=256, temperature=0.0, packed=packed, draft_cache=draft_cache)
    eng = Engine(cfg, DEV, pages=9, **args)
    prompts = ragged_prompts(cfg, lengths, 4)
    dims, model = parent_model(eng.weights["f16"])
    direct = eng.generate(prompts, max_new, routes=["f16"] * 4)
    for i, p in enumerate(prompts):
        gaps = check_greedy(dims, model, p, direct[i].tokens, f"f16 {i}")
        for route in ("int4", "fp8"):
            got = eng.generate([p], max_new, routes=[route])[0].tokens
            check_greedy(dims, model, p, got, f"{route} {i}")
            agree_until_near_tie(got, direct[i].tokens, gaps, f"{route} {i}")
    for d in eng.decoders.values():
        # as many pages as the rows' last positions need, each held once
        need = [-(-int(x) // 64) for x in d.pos_base.tolist()]
        assert int(d.pages.refs.sum()) == int(d.pages.held.sum()) and int(d.pages.refs.max()) == 1
        assert all(h >= n for h, n in zip(d.pages.held.tolist(), need)) and d.status.item() == 0


def test_graph_replays_are_the_eager_rounds():
    cfg = config(3)
    w = dec.DecoderWeights(cfg, DEV)
    prompts = ragged_prompts(cfg, [60, 127, 30], 6)
    uniforms = [(synth.uniform_u24((3, 3), 70 + r, DEV), synth.uniform_u24((3, 4), 90 + r, DEV)) for r in range(7)]
    outs = []
    for graph in (False, True):
        d = dec.SpecDecoder(w, capacity=256, temperature=0.9, pages=8, top_k=20, top_p=0.9)
        d.prefill_packed(prompts)
        for u in uniforms:
            d.set_uniforms(*u)
            if not graph:
                d.run()
            elif d.graph is None:
                d.capture()
            else:
                d.replay()
            torch.cuda.synchronize()
        assert d.status.item() == 0
        n = int(d.out_len.min())
        outs.append((d.out_len.tolist(), d.out_tokens[:, :n].cpu(), d.pages.held.tolist(), d.pages.table.tolist()))
    assert outs[0][0] == outs[1][0] and torch.equal(outs[0][1], outs[1][1]) and outs[0][2:] == outs[1][2:]
    assert min(outs[0][0]) >= 7 and max(outs[0][2]) >= 3  # (a page was taken within a replay)


@pytest.mark.parametrize("lengths,samples", [([130, 64], 3), ([65], 4), ([2, 129, 40], 2)])
def test_samples_share_their_prompts_pages(lengths, samples):
    cfg = config(len(lengths) * samples)
    w = dec.DecoderWeights(cfg, DEV)
    prompts = ragged_prompts(cfg, lengths, 8)
    own = sum(-(-(n - 1) // 64) for n in lengths)
    d = dec.DirectDecoder(w, capacity=256, temperature=0.0, pages=own + 3 * cfg.batch, samples=samples)
    d.prefill_packed(prompts)
    full = [(n - 1) // 64 for n in lengths]
    assert d.pages.refs.tolist().count(samples) == sum(full)
    part = sum((n - 1) % 64 > 0 for n in lengths)
    # a prompt's last page may lie past the entries that samples read
    assert int((d.pages.refs > 0).sum()) - sum(full) - part * samples in range(0, len(lengths) + 1)
    for _ in range(12):
        d.run()
    out = d.out_tokens[:, :12].tolist()
    assert d.status.item() == 0
    dims, model = parent_model(w)
    for g, p in enumerate(prompts):
        rows = out[g * samples:(g + 1) * samples]
        assert all(r == rows[0] for r in rows)
        check_greedy(dims, model, p, rows[0], f"prompt {g}")
    # different numbers, different continuations; the prompts' shared pages stay as they were
    d.T, d.filters = 1.0, dec.filter_rows(cfg.batch, 1.0, 50, 0.95, 0.0, DEV)
    d.prefill_packed(prompts)
    shared = (d.pages.refs == samples).nonzero()[:, 0]
    before = [a[:, shared].clone() for a in d.pcache.arrays]
    for r in range(10):
        d.set_uniforms(synth.uniform_u24((cfg.batch, 1), 200 + r, DEV))
        d.run()
    assert d.status.item() == 0
    assert all(torch.equal(a[:, shared], x) for a, x in zip(d.pcache.arrays, before))
    rows = d.out_tokens[:, :10].tolist()
    assert len({tuple(r) for r in rows[:samples]}) > 1


def test_tokens_of_filtered_draws():
    """The tokens are sq_sample_f32's definition over the decoder's own logits."""
    from test_gpu_sample import token

    cfg = config(4)
    w = dec.DecoderWeights(cfg, DEV)
    d = dec.DirectDecoder(w, capacity=128, temperature=0.8, pages=8, top_k=12, top_p=0.8, min_p=0.02)
    d.prefill_packed(ragged_prompts(cfg, [9, 30, 64, 65], 9))
    for r in range(6):
        u = synth.uniform_u24((4, 1), 300 + r, DEV)
        d.set_uniforms(u)
        d.run()
        rows = d.logits.cpu().numpy()
        assert d.next_token.tolist() == [token(rows[i], int(u[i, 0]), 0.8, 12, 0.8, 0.02) for i in range(4)]
    assert d.out_len.tolist() == [6] * 4 and d.status.item() == 0


@pytest.mark.parametrize("pages", [None, 12])
def test_rounds_emit_filtered_tokens(pages):
    cfg, k = config(3), 3
    w = dec.DecoderWeights(cfg, DEV)
    prompts = ragged_prompts(cfg, [20, 70, 33], 10)
    # top-1 of the parent is its greedy token, whatever is drafted
    one = dec.SpecDecoder(w, capacity=256, temperature=1.0, pages=pages, top_k=1)
    one.prefill_packed(prompts)
    for r in range(5):
        one.set_uniforms(synth.uniform_u24((k, 3), 400 + r, DEV), synth.uniform_u24((3, k + 1), 410 + r, DEV))
        one.run()
    dims, model = parent_model(w)
    for i, p in enumerate(prompts):
        check_greedy(dims, model, p, one.out_tokens[i, :int(one.out_len[i])].tolist(), f"sequence {i}")
    # what is emitted is among the tokens that the filters leave of the parent
    d = dec.SpecDecoder(w, capacity=256, temperature=1.0, pages=pages, top_k=5, top_p=0.9)
    d.prefill_packed(prompts)
    for r in range(6):
        start = d.out_len.tolist()
        d.set_uniforms(synth.uniform_u24((k, 3), 420 + r, DEV), synth.uniform_u24((3, k + 1), 430 + r, DEV))
        d.run()
        kept = d.target_logits > float("-inf")
        assert int(kept.sum(-1).max()) <= 5 and int((d.draft_logits > float("-inf")).sum(-1).max()) <= 5
        for i in range(3):
            emitted = d.out_tokens[i, start[i]:int(d.out_len[i])].tolist()
            assert emitted and all(bool(kept[i, j, t]) for j, t in enumerate(emitted))
    assert one.status.item() == 0 and d.status.item() == 0


def test_compaction_between_steps():
    """Moving the pages changes no token, and the pool's tail is free afterwards."""
    cfg = config(5)
    w = dec.DecoderWeights(cfg, DEV)
    prompts = ragged_prompts(cfg, [100, 64, 7, 190, 65], 11)
    outs = []
    for compact in (False, True):
        d = dec.SpecDecoder(w, batch=5, capacity=256, temperature=1.0, pages=40, draft_cache="q4")
        d.prefill_packed(prompts)
        for r in range(8):
            if r == 3:  # two sequences end, and others of their pages are taken by the rest
                keep = torch.tensor([-1, 0, -1, -1, 0], dtype=torch.int32, device=DEV)
                d.pages.trim(keep)
                d.pos_base.masked_fill_(keep == 0, -1)
            if compact and r in (4, 6):
                used = d.pages.compact([d.pcache, d.dcache], d.status)
                assert used == int((d.pages.refs > 0).sum()) and not d.pages.refs[used:].any()
                assert int(d.pages.table.max()) < used
            d.set_uniforms(synth.uniform_u24((3, 5), 500 + r, DEV), synth.uniform_u24((5, 4), 510 + r, DEV))
            d.run()
        outs.append([(int(d.out_len[i]), d.out_tokens[i, :int(d.out_len[i])].tolist()) for i in (0, 2, 3)])
    assert outs[0] == outs[1]


def test_a_pool_that_runs_out():
    """Rows without a page for their new entries emit nothing more and raise the status; the others go on as before."""
    cfg = config(2)
    w = dec.DecoderWeights(cfg, DEV)
    prompts = ragged_prompts(cfg, [40, 61], 12)
    d = dec.DirectDecoder(w, batch=2, capacity=256, temperature=0.0, pages=2)
    d.prefill_packed(prompts)
    for _ in range(20):
        d.run()
    assert d.status.item() & _lib.DEV_NO_PAGES and d.out_len.tolist() == [20, 4]
    dims, model = parent_model(w)
    for i, n in ((0, 20), (1, 4)):
        check_greedy(dims, model, prompts[i], d.out_tokens[i, :n].tolist(), f"sequence {i}")
    eng = Engine(cfg, DEV, layers=3, batch=2, capacity=256, pages=2, parent=w)
    with pytest.raises(RuntimeError, match="no token .*status flags"):
        eng.generate(prompts, 20, routes=["f16"] * 2)
    assert len(eng.generate(prompts, 3, routes=["f16"] * 2)[1].tokens) == 3  # the next requests fit
    # rows that have their tokens may run out while the others go on
    eng = Engine(cfg, DEV, layers=3, batch=2, capacity=256, pages=4, parent=w, k=3)
    got = [r.tokens for r in eng.generate(prompts, 40, routes=["int4"] * 2)]
    for i, p in enumerate(prompts):
        check_greedy(dims, model, p, got[i], f"request {i}")


def test_refusals():
    cfg = config(4)
    w = dec.DecoderWeights(cfg, DEV)
    for bad in (dict(pages=0), dict(pages=4, capacity=100), dict(pages=4, chains=2)):
        with pytest.raises(ValueError, match="paged caches"):
            dec.SpecDecoder(w, **{"capacity": 128, **bad})
    for bad in (dict(samples=3, pages=4), dict(samples=2)):
        with pytest.raises(ValueError, match="samples"):
            dec.DirectDecoder(w, capacity=128, **bad)
    for bad in (dict(top_p=float("nan")), dict(min_p=-1.0), dict(top_k=2.5)):
        with pytest.raises(ValueError, match="top_k"):
            dec.DirectDecoder(w, capacity=128, **bad)
    d = dec.DirectDecoder(w, capacity=128, pages=8, samples=2)
    prompts = ragged_prompts(cfg, [5, 6], 13)
    with pytest.raises(ValueError, match="prefill_packed"):
        d.prefill(padded(prompts), lengths=[5, 6])
    with pytest.raises(ValueError, match="group of samples"):
        d.prefill_packed(prompts * 2)
