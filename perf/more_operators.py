"""The calls over paged key/value caches and the sampling calls, as cases that can be timed and compared.

A cache of pages is a pool of pages of 64 positions per layer, a table of page ids per sequence, and a count of holders
per page, so that sequences share the pages of a common prefix.  A case is a dict of sizes; `prepare` makes what a program
holds before the call, `run` is one pass, `exact` the same result in 64 bits.

  attention  causal grouped-query attention of packed rows over pages: single tokens, blocks, prompts after a prefix
  rope       bias, rotation and the write of packed rows into pages; over 4-bit pages also the read of what was written
  fork       samples of a prompt: their rows released, forked from the prompt's, the pages of both halves copied in all
             layers, and room for the next tokens reserved
  compact    the used pages moved to the lowest ids, in the tables and in all layers
  sample     tokens drawn from logits with a temperature, top-k, top-p and min-p of each row's own
  filter     logits with the tokens that those filters drop set to -inf, as the acceptance of drafts takes them
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

HD = 128      # head dimension
GROUP = 64    # elements of a head's vector that share a scale and a zero
PAGE = 64     # positions of a page
THETA = 1e6

# Query and key/value heads and layers of the workloads in configs.py.
_1P5B = dict(hq=12, hkv=2)
_7B = dict(hq=28, hkv=4)
_VOCAB = 151936


def listed():
    return [
        # one conversation with a small model: latency
        dict(name="attn_f16_1p5b_1x1", kind="attention", cache="f16", b=1, lo=1, hi=1, past_lo=700, past_hi=700, shared=0,
             tail=0, mix=1, **_1P5B),
        # the next token of a batch of conversations, from short to very long
        dict(name="attn_f16_7b_64x1", kind="attention", cache="f16", b=64, lo=1, hi=1, past_lo=500, past_hi=24000, shared=0,
             tail=0, mix=2, **_7B),
        # prompts behind a long instruction whose pages they share
        dict(name="attn_f16_7b_prefix", kind="attention", cache="f16", b=8, lo=60, hi=900, past_lo=3011, past_hi=3011,
             shared=3008, tail=5, mix=3, **_7B),
        # a draft's step over 4-bit pages: the previous and the pending token of sixteen sequences
        dict(name="attn_q4_7b_16x2", kind="attention", cache="q4", b=16, lo=2, hi=2, past_lo=1000, past_hi=16000, shared=0,
             tail=0, mix=4, **_7B),
        # the new entries of a batch of single tokens
        dict(name="rope_f16_7b_64x1", kind="rope", cache="f16", b=64, lo=1, hi=1, past_lo=100, past_hi=9000, shared=0, tail=0,
             mix=5, **_7B),
        # ragged prompts into the 4-bit pages of a draft
        dict(name="rope_q4_7b_prompts", kind="rope", cache="q4", b=10, lo=30, hi=1500, past_lo=0, past_hi=0, shared=0, tail=3,
             mix=6, **_7B),
        # four samples of one prompt of a small model
        dict(name="fork_1p5b_1to4", kind="fork", layers=28, hkv=2, parents=1, children=4, len_lo=700, len_hi=700, ahead=1,
             mix=7),
        # eight samples of each of eight prompts
        dict(name="fork_7b_8to64", kind="fork", layers=28, hkv=4, parents=8, children=8, len_lo=300, len_hi=2500, ahead=9,
             mix=8),
        # a pool after many requests have come and gone
        dict(name="compact_7b", kind="compact", layers=28, hkv=4, rows=40, len_lo=60, len_hi=2000, spare=0.7, mix=9),
        # the next token of one request
        dict(name="sample_1", kind="sample", m=1, v=_VOCAB, ld=_VOCAB, spread=2.2, mix=10),
        # a batch of requests, each with settings of its own
        dict(name="sample_64", kind="sample", m=64, v=_VOCAB, ld=_VOCAB, spread=2.0, mix=11),
        # the parent's rows of a verification pass, before the acceptance: the head's rows are padded
        dict(name="filter_36", kind="filter", m=36, v=_VOCAB - 271, ld=_VOCAB, spread=2.0, mix=12),
    ]


# ------------------------------------------------------------------- draws
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    mix = rng.randrange(1 << 30)
    kind = rng.choice(["attention", "attention", "attention", "rope", "fork", "compact", "sample", "sample", "filter"])
    if kind in ("sample", "filter"):
        v = _log(rng, 500, 152000)
        m = _log(rng, 1, 96)
        return dict(kind=kind, m=m, v=v, ld=v + rng.choice([0, 0, rng.randint(1, 300)]),
                    spread=round(rng.uniform(0.3, 4.0), 2), mix=mix)
    hkv = rng.choice([1, 2, 4, 8])
    if kind == "fork":
        case = dict(kind=kind, layers=rng.randint(1, 32), hkv=hkv, parents=_log(rng, 1, 12), children=_log(rng, 1, 12),
                    len_lo=rng.randint(1, 200), len_hi=_log(rng, 200, 4000), ahead=rng.randint(1, 100), mix=mix)
        while work(case)["bytes"] > 5e8 or _pool_bytes(case) > 3e9:
            case["layers"] = max(1, case["layers"] // 2)
            case["children"] = max(1, case["children"] * 3 // 4)
            case["len_hi"] = max(200, case["len_hi"] * 3 // 4)
        return case
    if kind == "compact":
        case = dict(kind=kind, layers=rng.randint(1, 32), hkv=hkv, rows=_log(rng, 2, 60), len_lo=rng.randint(1, 60),
                    len_hi=_log(rng, 100, 3000), spare=round(rng.uniform(0.1, 1.0), 2), mix=mix)
        while work(case)["bytes"] > 9e8 or _pool_bytes(case) > 3e9:
            case["layers"] = max(1, case["layers"] // 2)
            case["rows"] = max(2, case["rows"] * 3 // 4)
        return case
    case = dict(kind=kind, cache=rng.choice(["f16", "q4"]), hq=hkv * rng.randint(1, min(10, 40 // hkv)), hkv=hkv, shared=0,
                tail=rng.randint(0, 9), mix=mix)
    form = rng.choice(["tokens", "tokens", "blocks", "prompts", "prefix"])
    if form == "tokens":
        hi = _log(rng, 64, 32000)
        case.update(b=_log(rng, 1, 96), lo=1, hi=rng.choice([1, 1, 2]), past_lo=rng.randint(0, hi), past_hi=hi)
    elif form == "blocks":
        rows, hi = rng.randint(3, 16), _log(rng, 64, 16000)
        case.update(b=_log(rng, 1, 16), lo=rows, hi=rows, past_lo=rng.randint(0, hi), past_hi=hi)
    elif form == "prompts":
        hi = _log(rng, 12, 3000)
        case.update(b=_log(rng, 1, max(1, min(32, 9000 // hi))), lo=rng.randint(1, hi), hi=hi, past_lo=0, past_hi=0)
    else:
        past = _log(rng, 64, 6000)
        case.update(b=_log(rng, 2, 10), lo=rng.randint(1, 40), hi=_log(rng, 41, 500), past_lo=past, past_hi=past,
                    shared=past // PAGE * PAGE)
    top = 0.9 * work(listed()[2])["flops"]
    while work(case)["flops"] > top or work(case)["bytes"] > 7e8:
        case["b"] = max(1, case["b"] // 2)
        case["past_hi"] = case["past_hi"] * 3 // 4
        case["past_lo"] = min(case["past_lo"], case["past_hi"])
        case["shared"] = min(case["shared"], case["past_lo"] // PAGE * PAGE)
    return case


def _layout(case):
    """Rows and cached positions of every sequence; from six sequences on, one has no rows."""
    rng = random.Random(case["mix"])
    lens = [_log(rng, case["lo"], case["hi"]) for _ in range(case["b"])]
    past = [_log(rng, case["past_lo"] + 1, case["past_hi"] + 1) - 1 for _ in range(case["b"])]
    if case["b"] >= 6 and case["lo"] < case["hi"]:
        lens[rng.randrange(case["b"])] = 0
    return lens, past


def _pages(n):
    return (n + PAGE - 1) // PAGE


def _tables(case):
    """Page ids of every sequence, scattered over the pool, and the pool's pages; a shared prefix holds the same ones."""
    lens, past = _layout(case)
    rng = random.Random(case["mix"] + 1)
    need = [_pages(n + p) for n, p in zip(lens, past)]
    common = case["shared"] // PAGE
    total = common + sum(n - common for n in need)
    ids = list(range(total + 3))
    rng.shuffle(ids)
    rows, at = [], common
    for n in need:
        rows.append(ids[:common] + ids[at:at + n - common])
        at += n - common
    return rows, total + 3


def _fork_layout(case):
    """(length, pages) of every parent and the parent of every child; rows: parents, then children."""
    rng = random.Random(case["mix"])
    lens = [_log(rng, case["len_lo"], case["len_hi"]) for _ in range(case["parents"])]
    lens = [n + (n % PAGE == 0) for n in lens]
    parent = [i for i in range(case["parents"]) for _ in range(case["children"])]
    ids = list(range(sum(_pages(n) for n in lens) + len(parent) * (2 + _pages(case["ahead"])) + 5))
    rng.shuffle(ids)
    tables = []
    for n in lens:
        tables.append(ids[:_pages(n)])
        ids = ids[_pages(n):]
    return lens, parent, tables, len(ids) + sum(len(t) for t in tables)


def _compact_layout(case):
    """Tables of sequences whose pages lie scattered over a pool, in pairs that share their first pages."""
    rng = random.Random(case["mix"])
    need = [_pages(_log(rng, case["len_lo"], case["len_hi"])) for _ in range(case["rows"])]
    pages = int(sum(need) * (1 + case["spare"])) + 2
    ids = list(range(pages))
    rng.shuffle(ids)
    tables = []
    for i, n in enumerate(need):
        common = tables[i - 1][:min(n, need[i - 1]) // 3] if i % 2 else []
        tables.append(common + ids[:n - len(common)])
        ids = ids[n - len(common):]
    return tables, pages


def _pool_bytes(case):
    pages = _fork_layout(case)[3] if case["kind"] == "fork" else _compact_layout(case)[1]
    return pages * case["layers"] * case["hkv"] * PAGE * HD * 4


def work(case):
    kind = case["kind"]
    if kind in ("sample", "filter"):
        n = case["m"] * case["v"]
        # the maximum, a weight and a comparison of every logit
        return {"bytes": 4 * n + (4 * n if kind == "filter" else 0) + 24 * case["m"], "flops": 4 * n}
    page = case["hkv"] * PAGE * HD * 4
    if kind == "fork":
        lens, parent, tables, pages = _fork_layout(case)
        copied = len(parent)
        held = 2 * sum(len(tables[p]) for p in parent)
        return {"bytes": 2 * copied * case["layers"] * page + 8 * held + 4 * pages, "flops": held}
    if kind == "compact":
        tables, pages = _compact_layout(case)
        used = {i for t in tables for i in t}
        moved = sum(i >= len(used) for i in used)
        held = sum(len(t) for t in tables)
        return {"bytes": 2 * moved * case["layers"] * page + 8 * held + 8 * pages, "flops": held + pages}
    lens, past = _layout(case)
    hq, hkv, rows = case["hq"], case["hkv"], sum(lens)
    entry = 2 * (HD // 2 + 4 * (HD // GROUP)) if case["cache"] == "q4" else 4 * HD  # a key and a value of one head
    if kind == "rope":
        n = rows * (hq + 2 * hkv) * HD * 4 + (hq + 2 * hkv) * HD * 2 + rows * hq * HD * 2 + rows * hkv * entry + 8 * rows
        if case["cache"] == "q4":
            n += rows * hkv * (entry + 4 * HD)
        return {"bytes": n, "flops": rows * (3 * (hq + hkv) + 2 * hkv) * HD}
    pairs = sum(n * p + n * (n + 1) // 2 for n, p in zip(lens, past))
    keys = case["shared"] + sum(n + p - case["shared"] for n, p in zip(lens, past) if n)
    return {"bytes": 2 * rows * hq * HD * 2 + keys * hkv * entry, "flops": 4 * HD * hq * pairs}


# ----------------------------------------------------------------- prepare
def _codes(w):
    """Codes 0 .. 15, scales and zeros of vectors [..., 128] fp16: groups of 64, the range widened to hold zero."""
    x = w.double().unflatten(-1, (-1, GROUP))
    lo, hi = x.amin(-1, keepdim=True).clamp(max=0), x.amax(-1, keepdim=True).clamp(min=0)
    flat = hi == lo
    want = torch.where(flat, 15.0, hi - lo) / 15
    s = want.float().half()
    s = torch.where(s.double() < want, (s.view(torch.int16) + 1).view(torch.float16), s).double()
    z = torch.where(flat, 0.0, torch.round(-lo / s).clamp(0, 15))
    q = (torch.round(x / s) + z).clamp(0, 15)
    v = (q - z) * s
    q = q - (v >= 65520).double() + (v <= -65520).double()  # a code stands for a finite binary16
    return q, s, z


def _swap(t, dim):
    """Index i of an axis at i with its two lowest bits exchanged."""
    i = torch.arange(t.shape[dim], device=t.device)
    return t.index_select(dim, (i & ~3) | ((i & 1) << 1) | ((i >> 1) & 1))


def _pack(k, v):
    """The 4-bit pages of keys and values [pages][hkv][64][128] fp16."""
    def half(w):
        q, s, z = _codes(w)
        byte = (q[..., 0, :] + 16 * q[..., 1, :]).to(torch.uint8)
        return byte, torch.cat([s[..., 0, :], z[..., 0, :], s[..., 1, :], z[..., 1, :]], -1).half()

    kq, ks = half(k)
    vq, vs = half(v)
    return (_swap(kq, 3).contiguous(), ks.contiguous(), _swap(vq.transpose(2, 3), 3).contiguous(),
            vs.transpose(2, 3).contiguous())


def _unpack(kq, ks, vq, vs):
    """Keys and values [pages][hkv][64][128] that 4-bit pages stand for, rounded to binary16, as fp32."""
    def values(byte, p):
        p = p.float()
        q = torch.cat([(byte & 15).float() - p[..., 1:2], (byte >> 4).float() - p[..., 3:4]], -1)
        return (q * torch.cat([p[..., 0:1].expand_as(byte), p[..., 2:3].expand_as(byte)], -1)).half().float()

    return values(_swap(kq, 3), ks), values(_swap(vq, 3).transpose(2, 3), vs.transpose(2, 3))


def _table(rows, width, dev):
    return torch.tensor([t + [-1] * (width - len(t)) for t in rows], dtype=torch.int32, device=dev)


def _holders(tables, pages, dev):
    n = [0] * pages
    for t in tables:
        for i in t:
            n[i] += 1
    return torch.tensor(n, dtype=torch.int32, device=dev)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=dev)

    kind = case["kind"]
    if kind in ("sample", "filter"):
        m, v, ld = case["m"], case["v"], case["ld"]
        x = normal(m, ld) * case["spread"]
        # the words that fit, some far above the others; every eighth row allows only part of the vocabulary
        hot = torch.randint(0, v, (m, 40), generator=g, device=dev)
        x.scatter_add_(1, hot, 8 * torch.rand(m, 40, generator=g, device=dev))
        banned = torch.rand(m, ld, generator=g, device=dev) < 0.3
        x = torch.where(banned & (torch.arange(m, device=dev) % 8 == 5)[:, None], torch.tensor(-math.inf, device=dev), x)
        rng = random.Random(case["mix"])
        settings = [(0.8, 50, 0.95, 0.0), (1.0, 0, 0.9, 0.0), (0.7, 0, 1.0, 0.05), (1.3, 200, 1.0, 0.0), (1.0, 0, 1.0, 0.0),
                    (0.0, 0, 1.0, 0.0), (1.5, 1000, 0.8, 0.02), (0.6, 20, 0.8, 0.1), (0.9, 0, 0.98, 0.01)]
        first = rng.randrange(len(settings)) if m > 1 else 0
        rows = [settings[(first + i) % len(settings)] for i in range(m)]
        st = dict(case=case, logits=x, u24=torch.randint(0, 1 << 24, (m,), generator=g, device=dev, dtype=torch.int32),
                  temperature=torch.tensor([r[0] for r in rows], device=dev), top_k=ints([r[1] for r in rows]),
                  top_p=torch.tensor([r[2] for r in rows], device=dev), min_p=torch.tensor([r[3] for r in rows], device=dev))
        st["out"] = torch.empty_like(x) if kind == "filter" else torch.empty(m, dtype=torch.int32, device=dev)
        if kind == "filter":
            st["out"].copy_(x)  # (what lies behind the vocabulary's end)
        return st

    if kind == "fork":
        lens, parent, tables, pages = _fork_layout(case)
        P, n = case["parents"], len(parent)
        width = max(_pages(x + case["ahead"]) for x in lens) + 1
        pool = (case["layers"], pages, case["hkv"])
        return dict(case=case, table=_table(tables + [[]] * n, width, dev), held=ints([len(t) for t in tables] + [0] * n),
                    refs=_holders(tables, pages, dev), parent=ints(parent), child=ints(list(range(P, P + n))),
                    length=ints([lens[p] for p in parent]), keep=ints([-1] * P + [0] * n),
                    pos=ints([-1] * P + [lens[p] for p in parent]), src=ints([0] * n), dst=ints([0] * n), count=ints([0]),
                    k=normal(*pool, PAGE, HD).half(), v=normal(*pool, HD, PAGE).half())

    if kind == "compact":
        tables, pages = _compact_layout(case)
        pool = (case["layers"], pages, case["hkv"])
        st = dict(case=case, table0=_table(tables, max(len(t) for t in tables) + 2, dev), held=ints([len(t) for t in tables]),
                  refs0=_holders(tables, pages, dev), src=ints([0] * pages), dst=ints([0] * pages), count=ints([0]),
                  used=ints([0]), k=normal(*pool, PAGE, HD).half(), v=normal(*pool, HD, PAGE).half())
        st["table"], st["refs"] = st["table0"].clone(), st["refs0"].clone()
        return st

    lens, past = _layout(case)
    tables, pages = _tables(case)
    b, hq, hkv = case["b"], case["hq"], case["hkv"]
    rows = sum(lens) + case["tail"]
    start = [0]
    for n in lens:
        start.append(start[-1] + n)
    st = dict(case=case, lens=lens, past=past, start=start, rows=rows, max_rows=max(lens), row_start=ints(start),
              pos=ints(past), tables=tables, table=_table(tables, max(len(t) for t in tables) + 1, dev))
    if kind == "rope":
        st["qkv"] = normal(rows, (hq + 2 * hkv) * HD)
        st["bias"] = (normal((hq + 2 * hkv) * HD) * 0.5).half()
        st["q_out"] = torch.zeros(rows, hq, HD, dtype=torch.float16, device=dev)
        f16, u8 = dict(dtype=torch.float16, device=dev), dict(dtype=torch.uint8, device=dev)
        if case["cache"] == "f16":
            st["cache"] = (torch.zeros(pages, hkv, PAGE, HD, **f16), torch.zeros(pages, hkv, HD, PAGE, **f16))
        else:
            st["cache"] = (torch.zeros(pages, hkv, PAGE, 64, **u8), torch.zeros(pages, hkv, PAGE, 4, **f16),
                           torch.zeros(pages, hkv, 64, PAGE, **u8), torch.zeros(pages, hkv, 4, PAGE, **f16))
            st["k_out"] = torch.zeros(rows, hkv, HD, **f16)
            st["v_out"] = torch.zeros(rows, hkv, HD, **f16)
        return st
    # queries a little larger than the keys, whose channels have offsets of their own; the first key draws weight
    st["q"] = (normal(rows, hq, HD) * 1.3).half()
    k = normal(pages, hkv, PAGE, HD) + normal(1, hkv, 1, HD) * 0.7
    first = sorted({t[0] for t in tables if t})
    k[first, :, 0] *= 2
    k = k.half()
    v = (normal(pages, hkv, PAGE, HD) + normal(1, hkv, 1, HD) * 0.5).half()
    st["cache"] = (k, v.transpose(2, 3).contiguous()) if case["cache"] == "f16" else _pack(k, v)
    st["out"] = torch.zeros(rows, hq, HD, dtype=torch.float16, device=dev)
    return st


# --------------------------------------------------------------------- run
def run(state):
    st, case = state, state["case"]
    kind = case["kind"]
    if not own:
        return {"attention": _plain_attention, "rope": _plain_rope, "fork": _plain_fork, "compact": _plain_compact,
                "sample": _plain_sample, "filter": _plain_filter}[kind](st)
    import paper_2609_21704_amd as sq

    if kind == "sample":
        return sq.sq_sample_f32(st["logits"], st["u24"], temperature=st["temperature"], top_k=st["top_k"],
                                top_p=st["top_p"], min_p=st["min_p"], vocab=case["v"], token=st["out"])
    if kind == "filter":
        return sq.sq_filter_logits_f32(st["logits"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"],
                                       min_p=st["min_p"], vocab=case["v"], out=st["out"])
    if kind == "fork":
        cache = (st["table"], st["held"], st["refs"])
        sq.sq_pages_trim(*cache, st["keep"])
        sq.sq_pages_fork(*cache, st["parent"], st["child"], st["length"], st["src"], st["dst"], st["count"])
        sq.sq_page_copy(st["k"], st["src"], st["dst"], st["count"])
        sq.sq_page_copy(st["v"], st["src"], st["dst"], st["count"])
        sq.sq_pages_reserve(*cache, st["pos"], case["ahead"])
        return {"table": st["table"], "held": st["held"], "refs": st["refs"], "k": st["k"], "v": st["v"]}
    if kind == "compact":
        st["table"].copy_(st["table0"])
        st["refs"].copy_(st["refs0"])
        sq.sq_pages_compact(st["table"], st["held"], st["refs"], st["src"], st["dst"], st["count"], st["used"])
        sq.sq_page_copy(st["k"], st["src"], st["dst"], st["count"])
        sq.sq_page_copy(st["v"], st["src"], st["dst"], st["count"])
        return {"table": st["table"], "refs": st["refs"], "used": st["used"], "k": st["k"], "v": st["v"]}
    rows = dict(max_rows=st["max_rows"])
    if kind == "rope":
        if case["cache"] == "f16":
            q = sq.sq_paged_rope_kv_f16(st["qkv"], st["bias"], st["row_start"], st["pos"], case["hq"], *st["cache"],
                                        st["table"], theta=THETA, q_out=st["q_out"], **rows)
            return {"q": q, "k": st["cache"][0], "v": st["cache"][1]}
        q = sq.sq_paged_rope_kv_q4(st["qkv"], st["bias"], st["row_start"], st["pos"], case["hq"], *st["cache"], st["table"],
                                   theta=THETA, q_out=st["q_out"], **rows)
        k, v = sq.sq_paged_kv_read_q4(*st["cache"], st["table"], st["row_start"], st["pos"], st["rows"], k_out=st["k_out"],
                                      v_out=st["v_out"], **rows)
        return {"q": q, "k": k, "v": v}
    call = sq.sq_paged_attention_f16 if case["cache"] == "f16" else sq.sq_paged_attention_q4
    return call(st["q"], *st["cache"], st["table"], st["row_start"], st["pos"], out=st["out"], **rows)


# ---- sampling
def _grid(v):
    """log2 of the weight of the likeliest token: the sum of v of them stays within 2^62."""
    return 62 - (v - 1).bit_length()


def _plain_kept(st):
    """Weights on the grid [m][v], int64, and which tokens the filters keep."""
    v = st["case"]["v"]
    x = st["logits"][:, :v]
    greedy = st["temperature"] == 0
    t = torch.where(greedy, 1.0, st["temperature"]).double()[:, None]
    z = x.double() / t  # (64 bits: whole numbers come of the weights)
    w = torch.exp(z - z.amax(-1, keepdim=True)).float()
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices
    ws = w.gather(1, order)
    r = torch.round(ws.double() * 2.0 ** _grid(v)).long()
    rank = torch.arange(v, device=x.device)
    k = torch.where((st["top_k"] > 0) & ~greedy, st["top_k"], v)
    k = torch.where(greedy, 1, k)
    kept = rank < k[:, None]
    rk = torch.where(kept, r, 0)
    need = torch.ceil(st["top_p"].double() * rk.sum(-1).double()).long().clamp(min=1)
    inside = (rk.cumsum(-1) - rk) < need[:, None]
    kept &= inside | (st["top_p"] >= 1)[:, None] | greedy[:, None]
    kept &= (ws >= st["min_p"].clamp(max=1)[:, None]) | greedy[:, None]
    weights = torch.empty_like(r).scatter_(1, order, r)
    return x, weights, torch.empty_like(kept).scatter_(1, order, kept)


def _plain_sample(st):
    _, r, kept = _plain_kept(st)
    c = torch.where(kept, r, 0).cumsum(-1)
    z, u = c[:, -1], st["u24"].long() & 0xFFFFFF
    t = u * (z >> 24) + ((u * (z & 0xFFFFFF)) >> 24)
    st["out"].copy_((c <= t[:, None]).sum(-1))
    return st["out"]


def _plain_filter(st):
    x, _, kept = _plain_kept(st)
    st["out"][:, :x.shape[1]] = torch.where(kept, x, torch.tensor(-math.inf, device=x.device))
    return st["out"]


# ---- pages
def _free(refs):
    return torch.sort((refs > 0).to(torch.uint8), stable=True).indices


def _add(refs, ids, n):
    refs.scatter_add_(0, ids.clamp(min=0).flatten().long(), torch.where(ids >= 0, n, 0).flatten().to(refs.dtype))


def _plain_copy(st, src, dst):
    for pool in (st["k"], st["v"]):
        pool[:, dst] = pool[:, src]


def _plain_fork(st):
    table, held, refs = st["table"], st["held"], st["refs"]
    i = torch.arange(table.shape[1], device=table.device)[None]
    # release
    want = torch.where(st["keep"] >= 0, (st["keep"] + PAGE - 1) // PAGE, held)
    drop = (i >= want[:, None]) & (i < held[:, None])
    _add(refs, torch.where(drop, table, -1), -1)
    table.masked_fill_(drop, -1)
    held.copy_(torch.minimum(held, want))
    # fork
    full, part = st["length"] // PAGE, st["length"] % PAGE > 0
    theirs = table[st["parent"].long()]
    rows = torch.where(i < full[:, None], theirs, -1)
    _add(refs, rows, 1)
    src = theirs.gather(1, full[:, None].long())[:, 0][part].long()
    dst = _free(refs)[:src.numel()]
    refs[dst] = 1
    fresh = torch.full_like(full, -1)
    fresh[part] = dst.to(fresh.dtype)
    rows = torch.where(i == full[:, None], fresh[:, None], rows)
    table[st["child"].long()] = rows
    held[st["child"].long()] = (full + part).to(held.dtype)
    _plain_copy(st, src, dst)
    # reserve
    want = torch.where(st["pos"] >= 0, (st["pos"] + st["case"]["ahead"] + PAGE - 1) // PAGE, held)
    new = (i >= held[:, None]) & (i < want[:, None])
    at = new.flatten().cumsum(0).view_as(new) - 1
    table.copy_(torch.where(new, _free(refs)[at.clamp(min=0)].to(table.dtype), table))
    _add(refs, torch.where(new, table, -1), 1)
    held.copy_(torch.maximum(held, want))
    return {"table": table, "held": held, "refs": refs, "k": st["k"], "v": st["v"]}


def _plain_compact(st):
    st["table"].copy_(st["table0"])
    st["refs"].copy_(st["refs0"])
    table, refs = st["table"], st["refs"]
    inside = refs > 0
    used = inside.sum()
    ids = torch.arange(refs.shape[0], device=refs.device)
    src, dst = ids[inside & (ids >= used)], ids[~inside & (ids < used)]
    to = ids.clone()
    to[src] = dst
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()], -1))
    refs[dst] = refs[src]
    refs[src] = 0
    st["used"].copy_(used)
    _plain_copy(st, src, dst)
    return {"table": table, "refs": refs, "used": st["used"], "k": st["k"], "v": st["v"]}


# ---- the paged cache
def _row_places(st, dev):
    """Position, page and place in the page of every packed row."""
    pos = torch.cat([torch.arange(p, p + n, device=dev) for n, p in zip(st["lens"], st["past"])])
    seq = torch.cat([torch.full((n,), i, device=dev) for i, n in enumerate(st["lens"])])
    return pos, st["table"][seq, pos // PAGE].long(), pos % PAGE


def _plain_rope(st):
    case, n = st["case"], st["start"][-1]
    hq, hkv = case["hq"], case["hkv"]
    u = (st["qkv"][:n] + st["bias"].float()).view(n, hq + 2 * hkv, HD)
    pos, page, at = _row_places(st, u.device)
    # positions times frequencies in 64 bits; the turn in 32, every product rounded
    t = torch.arange(64, device=u.device, dtype=torch.float64)
    angle = pos.double()[:, None] * torch.pow(torch.tensor(THETA, dtype=torch.float64), -t / 64)
    c, s = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    a, e = u[:, :hq + hkv, :64], u[:, :hq + hkv, 64:]
    turned = torch.cat([a * c - e * s, e * c + a * s], -1).half()
    q, k, v = turned[:, :hq], turned[:, hq:], u[:, hq + hkv:].half()
    st["q_out"][:n] = q
    if case["cache"] == "q4":
        for w, out in ((k, st["k_out"]), (v, st["v_out"])):
            code, scale, zero = _codes(w)
            out[:n] = ((code - zero) * scale).flatten(-2).float().half()
        return {"q": st["q_out"], "k": st["k_out"], "v": st["v_out"]}
    kc, vc = st["cache"]
    kc[page, :, at] = k
    vc[page, :, :, at] = v
    return {"q": st["q_out"], "k": kc, "v": vc}


def _plain_attention(st):
    case = st["case"]
    hq, hkv = case["hq"], case["hkv"]
    group = hq // hkv
    out = st["out"]
    for i, (n, p) in enumerate(zip(st["lens"], st["past"])):
        if n == 0:
            continue
        ids = st["table"][i, :_pages(n + p)].long()
        if case["cache"] == "f16":
            k, v = st["cache"][0][ids].float(), st["cache"][1][ids].transpose(2, 3).float()
        else:
            k, v = _unpack(*(c[ids] for c in st["cache"]))
        k, v = (x.transpose(0, 1).reshape(hkv, -1, HD)[:, :n + p] for x in (k, v))
        step = max(16, (1 << 28) // ((n + p + 1) * hq))  # rows whose scores are held at once
        for r in range(0, n, step):
            m = min(step, n - r)
            keys = p + r + m
            at = st["start"][i] + r
            q = st["q"][at:at + m].float().view(m, hkv, group, HD).permute(1, 0, 2, 3).reshape(hkv, m * group, HD)
            w = torch.matmul(q, k[:, :keys].transpose(1, 2).contiguous()) / math.sqrt(HD)
            last = p + r + torch.arange(m, device=q.device).repeat_interleave(group)
            w.masked_fill_(torch.arange(keys, device=q.device)[None, :] > last[:, None], float("-inf"))
            w -= w.amax(-1, keepdim=True)
            w.exp_()
            y = torch.matmul(w, v[:, :keys].contiguous()) / w.sum(-1, keepdim=True)
            out[at:at + m] = y.view(hkv, m, group, HD).permute(1, 0, 2, 3).reshape(m, hq, HD).half()
    return out


# ------------------------------------------------------------------- exact
def _exact_kept(case, st, row):
    """(logits, weights on the grid, kept) of one row, from the definition."""
    x = st["logits"][row, :case["v"]].cpu().numpy()
    temp = float(st["temperature"][row])
    if temp == 0:
        kept = np.zeros(x.size, bool)
        kept[int(np.argmax(x))] = True
        return x, kept.astype(np.int64), kept
    z = x.astype(np.float64) / temp
    w = np.exp(z - z.max()).astype(np.float32)
    r = np.rint(w.astype(np.float64) * 2.0 ** _grid(x.size)).astype(np.int64)
    order = np.lexsort((np.arange(x.size), -(x.astype(np.float64))))
    k = int(st["top_k"][row])
    if k > 0:
        order = order[:k]
    p = float(st["top_p"][row])
    if p < 1:
        run = np.cumsum(r[order])
        need = max(1, math.ceil(p * float(int(run[-1]))))
        order = order[:int(np.searchsorted(run - r[order], need))]  # the mass before them is less than the need
    kept = np.zeros(x.size, bool)
    kept[order] = True
    return x, r, kept & (w >= np.float32(min(1.0, float(st["min_p"][row]))))


def _exact_sample(case, st):
    tokens = []
    for row in range(case["m"]):
        _, r, kept = _exact_kept(case, st, row)
        ids = kept.nonzero()[0]
        run = np.cumsum(r[ids])
        t = ((int(st["u24"][row]) & 0xFFFFFF) * int(run[-1])) >> 24
        tokens.append(int(ids[np.searchsorted(run, t, side="right")]))
    return torch.tensor(tokens, dtype=torch.int32)


def _exact_filter(case, st):
    out = st["logits"].cpu().numpy().copy()
    for row in range(case["m"]):
        x, _, kept = _exact_kept(case, st, row)
        out[row, :x.size] = np.where(kept, x, -np.inf)
    return torch.from_numpy(out)


def _exact_fork(case, st):
    lens, parent, tables, pages = _fork_layout(case)
    refs = st["refs"].tolist()
    tables = [list(t) for t in tables]

    def take():
        i = min(j for j in range(pages) if refs[j] == 0)
        refs[i] = 1
        return i

    moves = []
    for p in parent:
        for j in tables[p][:lens[p] // PAGE]:
            refs[j] += 1
    for p in parent:
        t = tables[p][:lens[p] // PAGE]
        if lens[p] % PAGE:
            t.append(take())
            moves.append((tables[p][lens[p] // PAGE], t[-1]))
        tables.append(t)
    for c, p in enumerate(parent):
        t = tables[len(lens) + c]
        while len(t) * PAGE < lens[p] + case["ahead"]:
            t.append(take())
    k, v = st["k"].clone(), st["v"].clone()
    for a, b in moves:
        k[:, b], v[:, b] = st["k"][:, a], st["v"][:, a]
    dev = st["table"].device
    return {"table": _table(tables, st["table"].shape[1], dev), "held": torch.tensor([len(t) for t in tables]),
            "refs": torch.tensor(refs), "k": k, "v": v}


def _exact_compact(case, st):
    tables, pages = _compact_layout(case)
    refs = st["refs0"].tolist()
    used = sum(r > 0 for r in refs)
    holes = [j for j in range(used) if refs[j] == 0]
    to = {}
    for j in range(used, pages):
        if refs[j]:
            to[j] = holes[len(to)]
    k, v = st["k"].clone(), st["v"].clone()
    for a, b in to.items():
        refs[b], refs[a] = refs[a], 0
        k[:, b], v[:, b] = st["k"][:, a], st["v"][:, a]
    tables = [[to.get(j, j) for j in t] for t in tables]
    return {"table": _table(tables, st["table0"].shape[1], st["table0"].device), "refs": torch.tensor(refs),
            "used": torch.tensor([used]), "k": k, "v": v}


def _exact_rope(case, st):
    """Every entry from its formula; the 4-bit ones from keys and values at the precision the quantizer is given."""
    rows, hq, hkv, n = st["rows"], case["hq"], case["hkv"], st["start"][-1]
    x = st["qkv"].double().view(rows, -1, HD)[:n]
    x = (x + st["bias"].double().view(-1, HD)).float().double()
    where = torch.tensor([p + j for m, p in zip(st["lens"], st["past"]) for j in range(m)], dtype=torch.float64,
                         device=x.device)
    freq = torch.tensor([THETA ** (-t / 64) for t in range(64)], dtype=torch.float64, device=x.device)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=x.device), where[:, None] * freq)
    cos, sin = turn.real[:, None, :], turn.imag[:, None, :]
    lo, hi = x[..., :64], x[..., 64:]
    rot = torch.stack([lo * cos - hi * sin, hi * cos + lo * sin], 2).flatten(2)
    q = torch.zeros(rows, hq, HD, dtype=torch.float64, device=x.device)
    q[:n] = rot[:, :hq]
    if case["cache"] == "f16":
        pages = st["cache"][0].shape[0]
        k = torch.zeros(pages, hkv, PAGE, HD, dtype=torch.float64, device=x.device)
        v = torch.zeros(pages, hkv, HD, PAGE, dtype=torch.float64, device=x.device)
        for i, (m, p) in enumerate(zip(st["lens"], st["past"])):
            for page in range(p // PAGE, _pages(p + m)):  # the rows that lie in one page
                a, e = max(p, page * PAGE), min(p + m, (page + 1) * PAGE)
                rows_ = slice(st["start"][i] + a - p, st["start"][i] + e - p)
                at = slice(a - page * PAGE, e - page * PAGE)
                k[st["tables"][i][page], :, at] = rot[rows_, hq:hq + hkv].permute(1, 0, 2)
                v[st["tables"][i][page], :, :, at] = x[rows_, hq + hkv:].permute(1, 2, 0)
        return {"q": q, "k": k, "v": v}
    # what the codes stand for hangs on the rounding of the entries: fp32 cosines, sines, products and sums
    cf, sf = cos.float().double(), sin.float().double()

    def r32(t):
        return t.float().double()

    key = torch.stack([r32(r32(lo * cf) - r32(hi * sf)), r32(r32(hi * cf) + r32(lo * sf))], 2).flatten(2)[:, hq:hq + hkv]
    res = {"q": q}
    for name, w in (("k", key), ("v", x[:, hq + hkv:])):
        w = w.float().half().double().reshape(n, hkv, 2, GROUP)
        mn, mx = torch.clamp(w.min(-1).values, max=0.0), torch.clamp(w.max(-1).values, min=0.0)
        step = (mx - mn) / 15
        # the smallest binary16 not below it: its spacing is 2^(e - 10), 2^-24 below 2^-14
        e = torch.floor(torch.log2(torch.clamp(step, min=2.0 ** -40)))
        e = e + (torch.exp2(e + 1) <= step).double() - (torch.exp2(e) > step).double()
        ulp = torch.exp2(torch.clamp(e, min=-14.0) - 10)
        sc = torch.where(step > 0, torch.ceil(step / ulp) * ulp, torch.ones_like(step))[..., None]
        z = torch.clamp(torch.round(-mn[..., None] / sc), 0, 15)
        c = torch.clamp(torch.round(w / sc) + z, 0, 15) - z
        c = torch.where(torch.abs(c * sc) >= 65520, c - torch.sign(c), c)
        full = torch.zeros(rows, hkv, HD, dtype=torch.float64, device=x.device)
        full[:n] = (c * sc).reshape(n, hkv, HD)
        res[name] = full
    return res


def _exact_entries(codes, scales):
    """[64][128]: the binary16 values of one page's keys of a head, byte by byte as the layout is documented."""
    at = torch.tensor([4 * (i // 4) + (0, 2, 1, 3)[i % 4] for i in range(64)])
    codes = codes[:, at]
    low, high, s = (codes % 16).double(), (codes // 16).double(), scales.double()
    return torch.cat([(low - s[:, 1:2]) * s[:, 0:1], (high - s[:, 3:4]) * s[:, 2:3]], 1).float().half().double()


def _exact_attention(case, st):
    hq, hkv = case["hq"], case["hkv"]
    g = hq // hkv
    dev = st["q"].device
    out = torch.zeros(st["rows"], hq, HD, dtype=torch.float64, device=dev)
    if case["cache"] == "q4":
        at = torch.tensor([4 * (i // 4) + (0, 2, 1, 3)[i % 4] for i in range(64)])
        kc, ks, vc, vs = (c.cpu() for c in st["cache"])
        pages = range(kc.shape[0])
        keys = torch.stack([torch.stack([_exact_entries(kc[p, h], ks[p, h]) for h in range(hkv)]) for p in pages]).half()
        # a value's bytes: row j holds elements j and j + 64, the position's byte in exchanged order
        order = vc[:, :, :, at].permute(0, 1, 3, 2)
        vs = vs.permute(0, 1, 3, 2).double()
        low, high = (order % 16).double(), (order // 16).double()
        vals = torch.cat([(low - vs[..., 1:2]) * vs[..., 0:1], (high - vs[..., 3:4]) * vs[..., 2:3]], -1).float().half()
        keys, vals = keys.to(dev), vals.to(dev)
    else:
        keys, vals = st["cache"][0], st["cache"][1].transpose(2, 3)
    for i, (n, p) in enumerate(zip(st["lens"], st["past"])):
        if n == 0:
            continue
        for h in range(hkv):
            k = torch.cat([keys[j, h] for j in st["tables"][i]])[:p + n].double()
            v = torch.cat([vals[j, h] for j in st["tables"][i]])[:p + n].double()
            kt = k.t().contiguous()
            chunk = max(8, (1 << 26) // (p + n))
            for j in range(h * g, (h + 1) * g):
                for r in range(0, n, chunk):
                    m = min(chunk, n - r)
                    a = st["start"][i] + r
                    top = p + r + m
                    score = st["q"][a:a + m, j].double() @ kt[:, :top] * HD ** -0.5
                    allowed = torch.ones(m, top, dtype=torch.bool, device=dev).tril(p + r)
                    prob = torch.softmax(torch.where(allowed, score, torch.tensor(-math.inf, device=dev).double()), -1)
                    out[a:a + m, j] = prob @ v[:top]
    return out


def exact(case, seed):
    st = prepare(case, seed)
    return {"attention": _exact_attention, "rope": _exact_rope, "fork": _exact_fork, "compact": _exact_compact,
            "sample": _exact_sample, "filter": _exact_filter}[case["kind"]](case, st)
