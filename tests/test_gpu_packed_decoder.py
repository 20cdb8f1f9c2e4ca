"""GPU tests of the decoder and the engine over packed prompts and a 4-bit draft cache: packed against padded prompts, the
draft's pass over its 4-bit cache against one in 64 bits, and the engine's emitted tokens."""
import math

import pytest
import torch

from paper_2609_21704_amd import decoder as dec
from paper_2609_21704_amd import synth
from paper_2609_21704_amd.configs import CONFIGS, Config
from paper_2609_21704_amd.engine import Engine, cache_bytes
from test_gpu_engine import agree_until_near_tie, check_greedy, parent_model, ragged_prompts
from test_gpu_packed import quantized, values_q4

pytestmark = pytest.mark.gpu
DEV = "cuda"


def config(variant="int4", batch=3):
    return Config(0, "packed", 3, 512, 1152, 4, 2, 1000, variant, 2, batch, 5)


@pytest.mark.parametrize("variant,lengths,chains,rows", [("int4", [130, 2, 77], 1, 4096), ("fp8", [90, 41, 64], 1, 50),
                                                         ("int4", [70, 33], 2, 4096)])
def test_packed_prompts_fill_the_caches(monkeypatch, variant, lengths, chains, rows):
    monkeypatch.setattr(dec, "PREFILL_ROWS", rows)  # 50: prompts continue in the next pass
    cfg = config(variant, len(lengths))
    prompts = ragged_prompts(cfg, lengths, 3)
    w = dec.DecoderWeights(cfg, DEV)
    a, b = (dec.SpecDecoder(w, capacity=192, chains=chains) for _ in range(2))
    a.prefill_packed(prompts)
    padded = torch.zeros((len(lengths), max(lengths)), dtype=torch.int32)
    for i, p in enumerate(prompts):
        padded[i, :len(p)] = torch.tensor(p, dtype=torch.int32)
    b.prefill(padded, lengths=lengths)
    assert int(a.status.item()) == int(b.status.item()) == 0
    assert torch.equal(a.pending, b.pending) and torch.equal(a.prev, b.prev) and torch.equal(a.pos_base, b.pos_base)
    for x, y in ((a.dcache, b.dcache), (a.pcache, b.pcache)):
        for s, n in enumerate([n for n in lengths for _ in range(chains)]):
            for u, v in ((x.k_all[:, s, :, :n - 1], y.k_all[:, s, :, :n - 1]), (x.v_all[:, s, ..., :n - 1], y.v_all[:, s, ..., :n - 1])):
                # fp16 activations between the layers, and weights of the attention: roundings of 2^-11 differ
                assert float((u.double() - v.double()).norm() / v.double().norm()) <= 2e-3
            assert bool((x.k_all[:, s, :, n - 1:] == 0).all())  # nothing past the prompt
    with pytest.raises(ValueError, match="2 .. capacity"):
        a.prefill_packed(prompts[:-1] + [prompts[0][:1]])
    with pytest.raises(ValueError, match="one prompt"):
        a.prefill_packed(prompts[1:])


def draft_logits_64(d, prompt, block):
    """Logits of the draft's rows `block` after the prompt, in 64 bits from its dequantized weights, rounded to binary16
    where the layer rounds, keys and values to their 4-bit entries."""
    w, cfg, st = d.w, d.cfg, d.w.stack

    def f16(t):
        return t.half().double()

    def weight(key):
        c, s, z = st.draft[key]
        q = torch.stack([c & 15, c >> 4], -1).view(c.shape[0], -1, 128).double()
        return ((q - z.double()[..., None]) * s.double()[..., None]).view(c.shape[0], -1)

    def norm(h, g):
        return f16(h / torch.sqrt((h * h).mean(-1, keepdim=True) + dec.EPS) * g.double())

    toks = torch.tensor(list(prompt) + list(block), device=DEV)
    n, hd = toks.numel(), 128
    pos = torch.arange(n, device=DEV, dtype=torch.float64)
    ang = pos[:, None] * torch.pow(torch.tensor(dec.THETA, dtype=torch.float64), -torch.arange(64, device=DEV, dtype=torch.float64) / 64)
    cos, sin = torch.cos(ang)[:, None], torch.sin(ang)[:, None]

    def turn(x):
        lo, hi = x[..., :64], x[..., 64:]
        return f16(torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1))

    h = w.embed[toks].double()
    g = cfg.q_heads // cfg.kv_heads
    mask = torch.arange(n, device=DEV)[None] > torch.arange(n, device=DEV)[:, None]
    for l in range(w.layers):
        u = (norm(h, w.in_norm[l]) @ weight((l, "qkv")).t() + w.qkv_bias[l].double()).view(n, -1, hd)
        q = turn(u[:, :cfg.q_heads])
        k = quantized(turn(u[:, cfg.q_heads:cfg.q_heads + cfg.kv_heads]).half())[0].double()
        v = quantized(f16(u[:, cfg.q_heads + cfg.kv_heads:]).half())[0].double()
        a = torch.empty_like(q)
        for j in range(cfg.q_heads):
            s = (q[:, j] @ k[:, j // g].t().contiguous() / math.sqrt(hd)).masked_fill(mask, -math.inf)
            a[:, j] = f16(torch.softmax(s, -1) @ v[:, j // g])
        h = h + a.reshape(n, -1) @ weight((l, "o")).t()
        gate, up = (norm(h, w.post_norm[l]) @ weight((l, "gate_up")).t()).chunk(2, 1)
        h = h + f16(gate * torch.sigmoid(gate) * up) @ weight((l, "down")).t()
    return norm(h[len(prompt):], w.final_norm) @ weight((cfg.layers, "lm_head")).t()


@pytest.mark.parametrize("packed", [True, False])
def test_draft_pass_over_the_4_bit_cache(packed):
    cfg = config()
    lengths = [100, 5, 37]
    prompts = ragged_prompts(cfg, lengths, 7)
    d = dec.SpecDecoder(dec.DecoderWeights(cfg, DEV), capacity=192, draft_cache="q4")
    if packed:
        d.prefill_packed(prompts)
    else:
        padded = torch.zeros((3, 100), dtype=torch.int32)
        for i, p in enumerate(prompts):
            padded[i, :len(p)] = torch.tensor(p, dtype=torch.int32)
        d.prefill(padded, lengths=lengths)
    i32 = torch.int32
    block = torch.tensor([[p[-1], 11 + i, 500 + i] for i, p in enumerate(prompts)], dtype=i32, device=DEV)
    logits = torch.empty((9, cfg.vocab), device=DEV)
    d.forward(True, block[:, 0].contiguous(), block[:, 1:].t().contiguous(), 3, 0, logits, last_only=False)
    assert int(d.status.item()) == 0
    for i, p in enumerate(prompts):
        ref = draft_logits_64(d, p[:-1], block[i].tolist())
        got = logits.view(3, 3, -1)[i].double()
        # a 4-bit code of an entry at a border goes the other way now and then: a step of a sixteenth of its group
        assert float((got - ref).norm() / ref.norm()) <= 2e-2
    assert bool(torch.isfinite(values_q4(d.dcache.layer(0))[0].float()).all())


def test_refusals():
    w = dec.DecoderWeights(config(batch=2), DEV)
    with pytest.raises(ValueError, match="one chain"):
        dec.SpecDecoder(w, capacity=128, chains=2, draft_cache="q4")
    with pytest.raises(ValueError, match="one chain"):
        Engine(config(), DEV, chains=2, draft_cache="q4")
    with pytest.raises(ValueError, match="'f16' or 'q4'"):
        dec.SpecDecoder(w, capacity=128, draft_cache="int4")


@pytest.mark.parametrize("packed,draft_cache", [(True, "f16"), (True, "q4"), (False, "q4")])
def test_engine_emits_the_parents_tokens(packed, draft_cache):
    """Greedy requests over packed prompts and 4-bit draft caches: every emitted token is the parent's argmax (in 64 bits,
    up to a near tie), whatever the drafts were."""
    cfg = CONFIGS[1]
    eng = Engine(cfg, DEV, layers=2, k=3, batch=3, capacity=192, temperature=0.0, packed=packed, draft_cache=draft_cache)
    prompts = ragged_prompts(cfg, [40, 9, 77, 25], 23)
    out = eng.generate(prompts, 8, routes=["int4", "int4", "f16", "fp8"])
    dims, model = parent_model(eng.weights["f16"])
    for p, r in zip(prompts, out):
        check_greedy(dims, model, p, r.tokens, r.route)
    again = eng.generate(prompts, 8, routes=["int4", "int4", "f16", "fp8"])
    assert [r.tokens for r in again] == [r.tokens for r in out]


def test_cache_bytes_of_4_bits():
    cfg = CONFIGS[2]
    d = dec.KVCacheQ4(cfg, 2, 3, 128, DEV)
    have = sum(t.numel() * t.element_size() for t in (d.k_codes, d.k_scales, d.v_codes, d.v_scales))
    assert have == cache_bytes(cfg, 2, 3, 128, "q4") and cache_bytes(cfg, 2, 3, 128) == have * 512 // 144
