"""GPU checks of the packed attention at the far ends of its range: positions of millions beside short prompts, scores far
past fp32's whole numbers, weights to more than binary16, split keys of many sequences, prompts packed beside single tokens."""
import math

import pytest
import torch

import paper_2609_21704_amd as sq
from paper_2609_21704_amd.configs import Config
from paper_2609_21704_amd.decoder import DecoderWeights, SpecDecoder
from paper_2609_21704_amd.engine import Engine, weight_bytes
from test_gpu_packed import check_attention, ints, normal, pack_q4, starts, values_q4

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16 = torch.float16


@pytest.mark.parametrize("rows", [1, 0])
def test_a_prompt_beside_a_sequence_of_millions(rows):
    """A prompt's tiles beside a sequence (of one row, of none) 16.8 million positions on, 128 query heads on one: places in
    the order of the tiles are not all fp32 numbers, and every tile is taken."""
    hq, past, n = 128, 16_800_000, 601
    cap = past + 64
    c = (torch.zeros((2, 1, cap, 64), dtype=torch.uint8, device=DEV), torch.zeros((2, 1, cap, 4), dtype=F16, device=DEV),
         torch.zeros((2, 1, cap // 64, 64, 64), dtype=torch.uint8, device=DEV),
         torch.zeros((2, 1, cap // 64, 4, 64), dtype=F16, device=DEV))
    k, v = normal((1, 1, 640, 128), 111), normal((1, 1, 640, 128), 112)
    for t, x in zip(c, pack_q4(k, v)):
        t[1:, :, :x.shape[2]] = x
    q = normal((rows + n, hq, 128), 113, std=1.3)
    out = torch.full_like(q, 9.0)
    sq.sq_packed_attention_q4(q, *c, ints([0, rows, rows + n]), ints([past, 0]), max_rows=n, out=out)
    kd, vd = values_q4([t[1:, :, :640 if i < 2 else 10] for i, t in enumerate(c)])
    check_attention(out, q, kd, vd, [(n, 0)], lead=rows)
    assert bool((out[:rows] == 0).all())  # (its values are zeros)


@pytest.mark.parametrize("rows,past", [(1, 700), (4, 700), (9, 700), (150, 600), (30, 9000)])
@pytest.mark.parametrize("fmt", ["f16", "q4"])
def test_scores_past_whole_numbers_of_fp32(rows, past, fmt):
    """Scores up to 2.7e11, where neighbours in fp32 lie thousands apart.  Queries and keys of equal elements: a score is 128
    equal terms of at most 11 bits and a power of two, exact in fp32, so that the row's largest keys share the weight
    evenly and no other has any.  Then keys at random: the largest score takes all, wherever it leads by more than
    twice what 128 fp32 terms may be off (2^-24 each of the largest sum, and eight more roundings)."""
    hq, hkv, cap = 7, 1, 9088
    n = past + rows
    v = normal((1, hkv, cap, 128), 121)

    def run(q, k):
        if fmt == "f16":
            return sq.sq_packed_attention_f16(q, k, v.transpose(2, 3).contiguous(), starts([rows]), ints([past])), k, v
        cache = pack_q4(k, v)
        return sq.sq_packed_attention_q4(q, *cache, starts([rows]), ints([past])), *values_q4(cache)

    at = torch.arange(cap, device=DEV)
    for shape in ("up", "down", "steps"):
        c = {"up": at // 3, "down": (n - at).clamp(min=0) // 3, "steps": at * 37 % 11 * 100}[shape]
        c = (c.float() / c[:n].max() * 65504).clamp(max=65504).half()
        q = torch.full((rows, hq, 128), 32768.0, dtype=F16, device=DEV)
        out, kk, vv = run(q, c.view(1, 1, cap, 1).expand(1, hkv, cap, 128).contiguous())
        assert bool((kk == kk[..., :1]).all())
        seen = at[None, :n] <= past + torch.arange(rows, device=DEV)[:, None]
        s = torch.where(seen, kk[0, 0, :n, 0].double()[None], -math.inf)
        w = (s == s.amax(1, keepdim=True)).double()
        ref = (w @ vv[0, 0, :n].double()) / w.sum(1, keepdim=True)
        mag = (w @ vv[0, 0, :n].double().abs()) / w.sum(1, keepdim=True)
        # equal weights of 2^7 or a power of two below 2^15, sums of them in fp32, the output's rounding
        bound = ref.abs() * 2.0 ** -11 + mag * (n * 2.0 ** -24 + 2.0 ** -18) + 2.0 ** -25
        err = (out.double() - ref[:, None]).abs()
        assert bool((err <= bound[:, None]).all()), (shape, float(err.max()))
    q, k = normal((rows, hq, 128), 122, std=3000.0), normal((1, hkv, cap, 128), 123, std=3000.0)
    out, kk, vv = run(q, k)
    assert bool(torch.isfinite(out).all())
    s = torch.matmul(q.double().view(rows * hq, 128), kk[0, 0, :n].double().t().contiguous())
    s = s.masked_fill(at[None, :n] > (past + torch.arange(rows, device=DEV).repeat_interleave(hq))[:, None], -math.inf)
    top = s.topk(2, 1)
    dot = torch.matmul(q.double().abs().view(rows * hq, 128), kk[0, 0, :n].double().abs().t().contiguous()).amax(1)
    clear = top.values[:, 0] - top.values[:, 1] > 2 * dot * 136 * 2.0 ** -24 + 1000
    assert int(clear.sum()) > rows * hq // 2
    want = vv[0, 0, top.indices[:, 0][clear]].double()
    # a weight's binary16, the output's
    assert bool(((out.view(-1, 128)[clear].double() - want).abs() <= want.abs() * (2.0 ** -10 + 2.0 ** -18) + 2.0 ** -25).all())


@pytest.mark.parametrize("rows", [1, 4])
@pytest.mark.parametrize("past", [30, 5000])
def test_weights_of_few_rows_to_two_terms(rows, past):
    """Values whose weighted sum all but vanishes, so that the weights' roundings are seen beside the output's.  Scores are
    one product each, exact in fp32; the scale, the exponent's argument (below 32: 2^-20), the exponential and the
    sums come to 2^-18 of every weight, its two binary16 terms to 2^-20.  One binary16 would be 2^-12 off."""
    hq, hkv, cap = 7, 1, (past + rows + 63) // 64 * 64
    n = past + rows
    g = torch.Generator(device=DEV).manual_seed(131)
    k0 = torch.rand(n, generator=g, device=DEV) * 4 - 2
    k0[past:] = -30  # the block's own keys: hardly any weight, the same sum for all rows
    k0[:past][torch.arange(past, device=DEV) % (past // 30) != 0] = -30  # thirty keys have some
    k = torch.zeros((1, hkv, cap, 128), dtype=F16, device=DEV)
    k[0, 0, :n, 0] = k0.half()
    q = torch.zeros((rows, hq, 128), dtype=F16, device=DEV)
    q[..., 0] = 11.3125
    sign = torch.where(torch.rand(n, generator=g, device=DEV) < 0.5, 1.0, -1.0).double()
    w = torch.softmax(q[0, 0, 0].double() * k[0, 0, :past, 0].double() / math.sqrt(128), 0)
    value = (sign * (torch.rand(n, generator=g, device=DEV) * 0.7 + 0.35)).half()
    # some of the largest take away what is left of the sum, until it is about a rounding
    for i in torch.argsort(w, descending=True)[:6].tolist():
        left = float((w * value[:past].double()).sum() - w[i] * value[i].double())
        value[i] = -left / float(w[i])
    v = torch.zeros_like(k)
    v[0, 0, :n] = value[:, None]
    out = sq.sq_packed_attention_f16(q, k, v.transpose(2, 3).contiguous(), starts([rows]), ints([past]))
    kd, vd = k[0, 0, :n, 0].double(), v[0, 0, :n].double()
    s = q[0, 0, 0].double() * kd / math.sqrt(128)
    s = s.masked_fill(torch.arange(n, device=DEV)[None] > past + torch.arange(rows, device=DEV)[:, None], -math.inf)
    w = torch.softmax(s, 1)
    ref, mag = w @ vd, w @ vd.abs()
    bound = mag * (2.0 ** -18 + 2.0 ** -20) + n * 2.0 ** -32 * vd.abs().amax() + ref.abs() * 2.0 ** -11 + 2.0 ** -25
    err = (out.double() - ref[:, None]).abs()
    assert bool((err <= bound[:, None]).all()), float((err / bound[:, None]).max())


def test_engine_pads_where_no_projection_takes_packed_prompts():
    """Rows of 1184 elements, which no projection of many rows takes: the engine's packed prompts go padded, in blocks."""
    cfg = Config(0, "odd", 2, 512, 1184, 4, 2, 1000, "fp8", 2, 2, 5)
    tokens = []
    for packed in (True, False):
        w = DecoderWeights(cfg, DEV, variant="fp8")
        eng = Engine(cfg, DEV, batch=2, capacity=128, temperature=0.0, parent=w, packed=packed,
                     free_bytes=int(weight_bytes(cfg)["f16"] * 1.4) + (1 << 20))
        assert eng.plan["resident"] == ["f16"] and not eng.decoder("f16").takes_packed()
        tokens.append([r.tokens for r in eng.generate([[5, 6, 7], list(range(40)), [9, 1]], 6)])
    assert tokens[0] == tokens[1]
    d = SpecDecoder(w, batch=2, k=2, capacity=128)
    assert not d.takes_packed()
    with pytest.raises(ValueError, match="use prefill"):
        d.prefill_packed([[1, 2], [3, 4]])


# (rows, past) of more than 64 sequences on one kv head whose keys are split: single tokens with long caches below and above
# the 64th, empty ones between; few sequences with rows, of up to 70, among a hundred
MANY = [[((i % 5 != 2) * (1 + (i == 90)), 1100 * (i // 3 % 9) if i in (3, 70, 90, 119) else i % 60) for i in range(120)],
        [((40, 3000) if i == 2 else (33, 5000) if i == 66 else (70, 2000) if i == 99 else (0, 17 * i)) for i in range(100)]]


@pytest.mark.parametrize("seqs", MANY)
@pytest.mark.parametrize("fmt", ["f16", "q4"])
def test_split_keys_of_many_sequences(seqs, fmt):
    hq, hkv = 8, 1
    cap = (max(n + p for n, p in seqs) + 63) // 64 * 64
    b, rows, most = len(seqs), sum(n for n, _ in seqs), max(n for n, _ in seqs)
    q, k, v = normal((rows, hq, 128), 141, std=1.3), normal((b, hkv, cap, 128), 142), normal((b, hkv, cap, 128), 143)
    args = starts([n for n, _ in seqs]), ints([p for _, p in seqs])
    if fmt == "f16":
        out = sq.sq_packed_attention_f16(q, k, v.transpose(2, 3).contiguous(), *args, max_rows=most)
    else:
        cache = pack_q4(k, v)
        out = sq.sq_packed_attention_q4(q, *cache, *args, max_rows=most)
        k, v = values_q4(cache)
    check_attention(out, q, k, v, seqs)


@pytest.mark.parametrize("fmt", ["f16", "q4"])
def test_prompts_and_single_tokens_in_one_call(fmt):
    """A prompt packed beside single tokens after long caches; and the same in two calls over the same packed rows, whose
    row_start leaves the other sequences empty, each with a bound of its own."""
    hq, hkv, tokens = 28, 4, 9
    seqs = [(1, 700 + 450 * i) for i in range(tokens)] + [(500, 0), (60, 333)]
    cap = 4352
    b, rows = len(seqs), sum(n for n, _ in seqs)
    q, k, v = normal((rows, hq, 128), 151, std=1.3), normal((b, hkv, cap, 128), 152), normal((b, hkv, cap, 128), 153)
    start, pos = starts([n for n, _ in seqs]), ints([p for _, p in seqs])
    if fmt == "f16":
        cache, attn = (k, v.transpose(2, 3).contiguous()), sq.sq_packed_attention_f16
    else:
        cache, attn = pack_q4(k, v), sq.sq_packed_attention_q4
        k, v = values_q4(cache)
    check_attention(attn(q, *cache, start, pos, max_rows=500), q, k, v, seqs)
    out = torch.full_like(q, 9.0)
    attn(q, *cache, start.clamp(max=tokens), pos, max_rows=1, out=out)
    assert bool((out[tokens:] == 9).all())
    attn(q, *cache, start.clamp(min=tokens), pos, max_rows=500, out=out)
    check_attention(out, q, k, v, seqs)


@pytest.mark.parametrize("fmt", ["f16", "q4"])
def test_tiles_in_the_order_of_their_keys(fmt):
    """Eight sequences whose tiles do not run at once, two of them empty, some after cached positions: every row is there."""
    hq, hkv, seqs = 28, 4, [(1500, 0), (0, 900), (330, 40), (900, 0), (611, 200), (1203, 64), (0, 0), (1, 1700)]
    cap, b, rows = 1728, len(seqs), sum(n for n, _ in seqs)
    q, k, v = normal((rows, hq, 128), 161, std=1.3), normal((b, hkv, cap, 128), 162), normal((b, hkv, cap, 128), 163)
    args = starts([n for n, _ in seqs]), ints([p for _, p in seqs])
    if fmt == "f16":
        out = sq.sq_packed_attention_f16(q, k, v.transpose(2, 3).contiguous(), *args, max_rows=1500)
    else:
        cache = pack_q4(k, v)
        out = sq.sq_packed_attention_q4(q, *cache, *args, max_rows=1500)
        k, v = values_q4(cache)
    check_attention(out, q, k, v, seqs)


@pytest.mark.parametrize("rows,past", [(1, 90), (4, 200), (40, 300)])
@pytest.mark.parametrize("fmt", ["f16", "q4"])
def test_infinite_values_that_every_row_reads(rows, past, fmt):
    """An infinite value below every row's position, at the key of the largest score (a weight that is one binary16 alone)
    and at others: the outputs are infinite in its dimension, and nowhere else."""
    hq, hkv, cap = 7, 1, 384
    q, k, v = normal((rows, hq, 128), 171), normal((1, hkv, cap, 128), 172), normal((1, hkv, cap, 128), 173)
    k[..., 0] = 0
    q[..., 0] = 8.0
    k[0, 0, 7, 0] = 10.0
    for key in (7, 3):
        if fmt == "f16":
            args = starts([rows]), ints([past])
            clean = sq.sq_packed_attention_f16(q, k, v.transpose(2, 3).contiguous(), *args)
            w = v.clone()
            w[0, 0, key, 5], w[0, 0, key, 70] = math.inf, -math.inf
            out = sq.sq_packed_attention_f16(q, k, w.transpose(2, 3).contiguous(), *args)
            hit = torch.zeros(128, device=DEV)
            hit[5], hit[70] = math.inf, -math.inf
        else:
            cache = pack_q4(k, v)
            clean = sq.sq_packed_attention_q4(q, *cache, starts([rows]), ints([past]))
            vs = cache[3].clone()
            vs[0, 0, 0, 2, key] = math.inf  # elements 64 .. 127 of one value: a zero of 7.5 lies between codes
            vs[0, 0, 0, 3, key] = 7.5
            out = sq.sq_packed_attention_q4(q, *cache[:3], vs, starts([rows]), ints([past]))
            hit = torch.zeros(128, device=DEV)
            c = cache[2][0, 0, 0, :, (key & ~3) | ((key & 1) << 1) | ((key >> 1) & 1)] >> 4
            hit[64:] = torch.where(c > 7, math.inf, -math.inf)
        want = torch.where(hit == 0, clean.float(), hit.expand_as(clean))
        assert torch.equal(out.float(), want), key
