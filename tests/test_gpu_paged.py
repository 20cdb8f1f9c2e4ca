"""GPU checks of the calls over paged caches (include/specquant_paged.h): the rotation and write against the calls over
contiguous caches, the attention against a 64-bit softmax and those calls, at lengths from none to thousands, pages that
sequences share, odd sizes, every kernel and key split, entries outside the pool, stale and non-finite entries."""
import math
import random

import pytest
import torch

import paper_2609_21704_amd as sq
from paper_2609_21704_amd import _lib, synth

pytestmark = pytest.mark.gpu
DEV = "cuda"
NAN = float("nan")
I32, F16, U8 = torch.int32, torch.float16, torch.uint8


def normal(shape, *seed, std=1.0):
    return synth.normal_f16(shape, std, synth.stream_seed(83, *seed), torch.device(DEV))


def ints(v):
    return torch.tensor(v, dtype=I32, device=DEV)


def starts(lens, lead=0):
    s = [lead]
    for n in lens:
        s.append(s[-1] + n)
    return ints(s)


def tables(lens, seed, spare=3, extra=2, shared=0):
    """Page ids [b][width] scattered over a pool for sequences of these lengths, and the pool's pages; the first `shared`
    pages of every sequence are the same."""
    rng = random.Random(seed)
    need = [(n + 63) // 64 for n in lens]
    total = shared + sum(max(0, n - shared) for n in need) + spare
    ids = rng.sample(range(total), total)
    common, ids = ids[:shared], ids[shared:]
    width, rows = max(need) + extra, []
    for n in need:
        k = max(0, n - shared)
        rows.append(common[:n] + ids[:k] + [-1] * (width - n))
        ids = ids[k:]
    return ints(rows), total


def nan_pool(pages, hkv, q4):
    if not q4:
        return (torch.full((pages, hkv, 64, 128), NAN, dtype=F16, device=DEV),
                torch.full((pages, hkv, 128, 64), NAN, dtype=F16, device=DEV))
    return (torch.full((pages, hkv, 64, 64), 0xA5, dtype=U8, device=DEV),
            torch.full((pages, hkv, 64, 4), NAN, dtype=F16, device=DEV),
            torch.full((pages, hkv, 64, 64), 0x5A, dtype=U8, device=DEV),
            torch.full((pages, hkv, 4, 64), NAN, dtype=F16, device=DEV))


def to_pages(cache, table, pages):
    """The pool that holds the entries of a contiguous cache; entries of no page are garbage."""
    q4 = len(cache) == 4
    b, hkv, cap = cache[0].shape[:3]
    pool = nan_pool(pages, hkv, q4)
    for s in range(b):
        for i, page in enumerate(table[s, :cap // 64].tolist()):
            if page < 0:
                continue
            at = slice(64 * i, 64 * i + 64)
            if q4:
                parts = cache[0][s, :, at], cache[1][s, :, at], cache[2][s, :, i], cache[3][s, :, i]
            else:
                parts = cache[0][s, :, at], cache[1][s, :, :, at]
            for p, x in zip(pool, parts):
                p[page] = x
    return pool


def calls(q4):
    if q4:
        return sq.sq_paged_rope_kv_q4, sq.sq_packed_rope_kv_q4, sq.sq_paged_attention_q4, sq.sq_packed_attention_q4
    return sq.sq_paged_rope_kv_f16, sq.sq_packed_rope_kv_f16, sq.sq_paged_attention_f16, sq.sq_packed_attention_f16


def bits(t):
    return t.view(torch.int16) if t.dtype == F16 else t


# (rows, past) per sequence, hq, hkv, rows before and after them
ROWS = [([(1, 0)], 4, 4, 0, 0),
        ([(1, 63), (1, 64)], 7, 1, 0, 0),
        ([(2, 1), (0, 5), (2, 126)], 28, 4, 1, 2),
        ([(17, 3), (1, 0), (0, 0), (40, 0), (16, 16), (5, 59)], 12, 2, 2, 3),
        ([(300, 0), (33, 1000), (129, 7)], 8, 8, 0, 5),
        ([(1, i % 60) for i in range(150)], 3, 1, 0, 1)]


@pytest.mark.parametrize("seqs,hq,hkv,lead,tail", ROWS)
@pytest.mark.parametrize("q4", [False, True])
def test_rope_write(seqs, hq, hkv, lead, tail, q4):
    """The bits of the call over a contiguous cache, at the positions' pages; nothing else is written."""
    paged, packed, _, _ = calls(q4)
    b, lens, past = len(seqs), [n for n, _ in seqs], [p for _, p in seqs]
    rows, ends = lead + sum(lens) + tail, [n + p for n, p in seqs]
    table, pages = tables(ends, rows)
    cap = 64 * table.shape[1]
    qkv = normal((rows, (hq + 2 * hkv) * 128), 1, rows).float() * 1.37
    bias = normal(((hq + 2 * hkv) * 128,), 2, hq)
    start, pos = starts(lens, lead), ints([p - 5 for p in past])
    args = dict(max_rows=max(lens), pos_offset=5)
    status = torch.zeros(1, dtype=I32, device=DEV)
    if q4:
        cache = (torch.full((b, hkv, cap, 64), 0xA5, dtype=U8, device=DEV),
                 torch.full((b, hkv, cap, 4), NAN, dtype=F16, device=DEV),
                 torch.full((b, hkv, cap // 64, 64, 64), 0x5A, dtype=U8, device=DEV),
                 torch.full((b, hkv, cap // 64, 4, 64), NAN, dtype=F16, device=DEV))
    else:
        cache = (torch.full((b, hkv, cap, 128), NAN, dtype=F16, device=DEV),
                 torch.full((b, hkv, 128, cap), NAN, dtype=F16, device=DEV))
    q0, q1 = (torch.full((rows, hq, 128), 9.0, dtype=F16, device=DEV) for _ in range(2))
    packed(qkv, bias, start, pos, hq, *cache, q_out=q0, **args)
    pool = nan_pool(pages, hkv, q4)
    paged(qkv, bias, start, pos, hq, *pool, table, q_out=q1, status=status, **args)
    assert torch.equal(q0, q1) and int(status) == 0
    for got, want in zip(pool, to_pages(cache, table, pages)):
        assert torch.equal(bits(got), bits(want))
    if q4:
        want = sq.sq_packed_kv_read_q4(*cache, start, pos, rows, **args)
        got = sq.sq_paged_kv_read_q4(*pool, table, start, pos, rows, k_out=torch.zeros_like(want[0]),
                                     v_out=torch.zeros_like(want[1]), **args)
        inside = slice(lead, lead + sum(lens))
        for g, w in zip(got, want):
            assert torch.equal(bits(g[inside]), bits(w[inside])) and not g[:lead].any() and not g[inside.stop:].any()


def exact(q, k, v, lens, past, start):
    """[rows][hq][128] fp64 and the same weighted means of |v|; k, v: per sequence [hkv][keys][128]."""
    hq = q.shape[1]
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    for i, (n, p) in enumerate(zip(lens, past)):
        hkv = k[i].shape[0]
        for j in range(hq):
            h = j // (hq // hkv)
            rows = slice(start[i], start[i] + n)
            s = q[rows, j].double() @ k[i][h].double().t().contiguous() / math.sqrt(128)
            last = p + torch.arange(n, device=DEV)[:, None]
            s = s.masked_fill(torch.arange(n + p, device=DEV)[None] > last, -math.inf)
            out[rows, j] = torch.softmax(s, -1) @ v[i][h].double()
    return out


# rows and past of every sequence; hq, hkv; shared pages: single tokens, blocks, turns, prompts, a shared prefix; few and
# many sequences (whole and split keys), lengths that differ much
ATTN = [([(1, 0)], 1, 1, 0),
        ([(1, 700)], 12, 2, 0),
        ([(1, 63), (1, 64), (1, 127), (0, 0), (1, 0)], 28, 4, 1),
        ([(1, 30 + 37 * i) for i in range(40)], 28, 4, 0),
        ([(1, 5000), (1, 3), (1, 900)], 8, 8, 0),
        ([(1, 20 * (i % 7) ** 3) for i in range(70)], 8, 4, 0),
        ([(1, 30000)] + [(1, 10 + i) for i in range(34)], 8, 4, 0),
        ([(2, (i * 797) % 3100) for i in range(150)], 14, 2, 0),
        ([(i % 3, 70 * (i % 9)) for i in range(70)], 16, 4, 1),
        ([(5, 90 * (i % 11)) for i in range(66)], 24, 4, 0),
        ([(2, 640 * i) for i in range(9)], 28, 4, 0),
        ([(9, 200), (9, 1900), (9, 0), (9, 64)], 28, 4, 1),
        ([(16, 100 * i) for i in range(20)], 8, 2, 0),
        ([(40, 4000), (17, 3000)], 28, 4, 40),
        ([(300, 0), (0, 0), (65, 0), (1, 0), (128, 0)], 12, 2, 0),
        ([(100, 1000), (33, 1000), (250, 1000), (64, 1000)], 28, 4, 15),
        ([(1300, 0), (700, 3)], 40, 8, 0)]


def pool_of(table, pages, lens, past, hkv, q4, seed):
    """A pool with random entries in the sequences' pages, NaN in the others, and the keys and values by sequence."""
    k, v = normal((pages, hkv, 64, 128), 3, seed), normal((pages, hkv, 64, 128), 4, seed)
    k[table[0, 0].clamp(min=0)][:, 0] *= 2
    used = sorted({i for row, n, p in zip(table.tolist(), lens, past) for i in row[:(n + p + 63) // 64]})
    if q4:
        pool = nan_pool(pages, hkv, True)
        # through the write: a sequence a page, at its 64 positions
        one = ints([[i] for i in used])
        qkv = torch.cat([torch.zeros_like(k), k, v], 1)[used].permute(0, 2, 1, 3).reshape(len(used) * 64, -1).float()
        sq.sq_paged_rope_kv_q4(qkv.contiguous(), None, None, ints([0] * len(used)), hkv, *pool, one, max_rows=64)
        ko, vo = sq.sq_paged_kv_read_q4(*pool, one, None, ints([0] * len(used)), len(used) * 64, max_rows=64)
        k[used] = ko.view(len(used), 64, hkv, 128).transpose(1, 2)
        v[used] = vo.view(len(used), 64, hkv, 128).transpose(1, 2)
    else:
        stale = [i for i in range(pages) if i not in used]
        k[stale], v[stale] = NAN, NAN
        pool = (k, v.transpose(2, 3).contiguous())
    by_seq = [[torch.cat([x[i] for i in row[:(n + p + 63) // 64]], 1)[:, :n + p] if n + p else x[0, :, :0]
               for row, n, p in zip(table.tolist(), lens, past)] for x in (k, v)]
    return pool, by_seq


def check_attention(out, ref, by_seq, hq, two_terms):
    """Per element: the output's rounding 2^-11 |o|; a weight's rounding, 2^-11 of itself in one term and 2^-20 in two, by
    sum w |v| <= max |v|; scores, exponentials and sums in fp32, a few 2^-20 of max |v|."""
    top = max([float(v.abs().max()) for v in by_seq if v.numel()] + [0.0])
    tol = 2.0 ** -11 * ref.abs() + (2.0 ** -11 * (not two_terms) + 2.0 ** -16) * top + 2.0 ** -24
    err = (out.double() - ref).abs()
    assert bool((err <= tol).all()), float((err / tol).max())


@pytest.mark.parametrize("seqs,hq,hkv,shared", ATTN)
@pytest.mark.parametrize("q4", [False, True])
def test_attention(seqs, hq, hkv, shared, q4):
    lens, past = [n for n, _ in seqs], [p for _, p in seqs]
    ends = [n + p for n, p in seqs]
    table, pages = tables(ends, len(seqs), shared=shared)
    pool, (k, v) = pool_of(table, pages, lens, past, hkv, q4, len(seqs))
    rows = sum(lens) + 3
    q = normal((rows, hq, 128), 5, rows, std=1.3)
    start, pos = starts(lens, 1), ints([p + 2 for p in past])
    out = torch.full((rows, hq, 128), 7.0, dtype=F16, device=DEV)
    args = dict(max_rows=max(lens), pos_offset=-2, len_bound=max(ends))
    calls(q4)[2](q, *pool, table, start, pos, out=out, **args)
    assert bool((out[0] == 7).all()) and bool((out[rows - 2:] == 7).all())  # rows of no sequence
    ref = exact(q, k, v, lens, past, start.tolist())
    inside = slice(1, 1 + sum(lens))
    check_attention(out[inside], ref[inside], v, hq, not q4 and max(lens) * (hq // hkv) <= 32)
    again = calls(q4)[2](q, *pool, table, start, pos, **args)
    assert torch.equal(again[inside], out[inside])


@pytest.mark.parametrize("seqs,hq,hkv", [([(1, 700), (1, 0), (1, 5000)], 28, 4), ([(2, 300)] * 5, 8, 8),
                                         ([(1, 30 * i) for i in range(40)], 28, 4), ([(9, 1000), (9, 77)], 28, 4),
                                         ([(40, 4000)], 28, 4), ([(300, 0), (129, 64), (0, 3)], 12, 2)])
@pytest.mark.parametrize("q4", [False, True])
def test_the_bits_of_contiguous_caches(seqs, hq, hkv, q4):
    """The attention over a contiguous cache with the same entries, wherever the sequences' keys are split as there."""
    lens, past = [n for n, _ in seqs], [p for _, p in seqs]
    table, pages = tables([n + p for n, p in seqs], 31)
    pool, _ = pool_of(table, pages, lens, past, hkv, q4, 32)
    ids = table.clamp(min=0).long()  # (entries of no page are never read)
    if q4:
        whole = [pool[0][ids].permute(0, 2, 1, 3, 4).flatten(2, 3), pool[1][ids].permute(0, 2, 1, 3, 4).flatten(2, 3),
                 pool[2][ids].transpose(1, 2), pool[3][ids].transpose(1, 2)]
    else:
        whole = [pool[0][ids].permute(0, 2, 1, 3, 4).flatten(2, 3), pool[1][ids].permute(0, 2, 3, 1, 4).flatten(3, 4)]
    rows = sum(lens)
    q = normal((rows, hq, 128), 33, rows)
    args = dict(max_rows=max(lens), len_bound=max(n + p for n, p in seqs))
    got = calls(q4)[2](q, *pool, table, starts(lens), ints(past), **args)
    want = calls(q4)[3](q, *[x.contiguous() for x in whole], starts(lens), ints(past), **args)
    if 2 * len(seqs) * hkv > 256 and max(lens) * (hq // hkv) <= (64 if q4 else 32):  # cut into equal shares instead
        assert float((got.double() - want.double()).abs().max()) <= 2.0 ** -9 * float(want.abs().max())
    else:
        assert torch.equal(got, want)


@pytest.mark.parametrize("rows", [1, 2, 9, 130])
@pytest.mark.parametrize("q4", [False, True])
def test_offsets_past_32_bits(rows, q4):
    """Pages whose bytes lie beyond 4 GiB of a pool's array: as the same pages at its start."""
    hq, hkv, past = 16, 8, [500, 63]
    paged_rope, _, paged, _ = calls(q4)
    pages = 140000 if q4 else 40000
    small, n = tables([p + rows for p in past], 41, spare=0, extra=0)
    pool = nan_pool(n, hkv, q4)
    far = [torch.empty((pages, *x.shape[1:]), dtype=x.dtype, device=DEV) for x in pool]
    assert far[0].numel() * far[0].element_size() > 1 << 32
    shift = pages - n
    for x, y in zip(pool, far):
        y[shift:] = x  # (what no position writes)
    big = torch.where(small >= 0, small + shift, small)
    # all positions written, then the last ones once more with their queries
    ends = [p + rows for p in past]
    qkv = normal((sum(ends), (hq + 2 * hkv) * 128), 42, rows).float()
    new = normal((2 * rows, (hq + 2 * hkv) * 128), 43, rows).float()
    outs = []
    for cache, table in ((pool, small), (far, big)):
        paged_rope(qkv, None, starts(ends), ints([0, 0]), hq, *cache, table, max_rows=max(ends))
        q = paged_rope(new, None, None, ints(past), hq, *cache, table, max_rows=rows)
        outs.append(paged(q, *cache, table, None, ints(past), max_rows=rows))
    assert torch.equal(outs[0], outs[1]) and bool(torch.isfinite(outs[0]).all())
    used = sorted({i for row in small.tolist() for i in row if i >= 0})
    for x, y in zip(pool, far):
        assert torch.equal(bits(x[used]), bits(y[shift:][used]))


def test_a_list_of_steps_past_32_bits():
    """So many and such wide rows that the bound of their steps counts several as one."""
    hq, hkv, b, width = 8, 4, 300, 1 << 20
    past = [(i * 37) % 1500 for i in range(b)]
    small, pages = tables([p + 1 for p in past], 51, extra=0)
    pool, (k, v) = pool_of(small, pages, [1] * b, past, hkv, False, 52)
    table = torch.full((b, width), -1, dtype=I32, device=DEV)
    table[:, :small.shape[1]] = small
    q = normal((b, hq, 128), 53)
    out = sq.sq_paged_attention_f16(q, *pool, table, None, ints(past), max_rows=1)
    check_attention(out, exact(q, k, v, [1] * b, past, list(range(b))), v, hq, True)


@pytest.mark.parametrize("rows,hq,hkv", [(1, 28, 4), (2, 28, 4), (9, 28, 4), (9, 8, 8), (100, 12, 2)])
@pytest.mark.parametrize("q4", [False, True])
def test_pages_outside_the_pool(rows, hq, hkv, q4):
    """Rows that read a position of no page are NaN, the others as without it; nothing is written there."""
    paged_rope, _, paged, _ = calls(q4)
    past = [0, 130, 64, 300]
    lens, ends = [rows] * 4, [rows + p for p in past]
    table, pages = tables(ends, 5, extra=0)
    pool, _ = pool_of(table, pages, lens, past, hkv, q4, 6)
    q = normal((4 * rows, hq, 128), 7, rows)
    args = dict(max_rows=rows, len_bound=max(ends))
    good = paged(q, *pool, table, None, ints(past), **args)
    bad = table.clone()
    bad[1, 1], bad[2, (64 + rows - 1) // 64], bad[3, 0] = pages, -1, -2 ** 31
    out = paged(q, *pool, bad, None, ints(past), **args)
    for s, first in ((0, 10 ** 6), (1, 64), (2, (64 + rows - 1) // 64 * 64), (3, 0)):
        for j in range(rows):
            got = out[s * rows + j]
            if past[s] + j >= first:
                assert bool(torch.isnan(got).all()), (s, j)
            else:
                assert torch.equal(got, good[s * rows + j]), (s, j)
    # the write: a sequence whose new rows have no page
    qkv = normal((4 * rows, (hq + 2 * hkv) * 128), 8, rows).float()
    status = torch.zeros(1, dtype=I32, device=DEV)
    none = table.clone()
    none[2] = pages + 3
    a, b = [x.clone() for x in pool], [x.clone() for x in pool]
    qa = paged_rope(qkv, None, None, ints(past), hq, *a, table, status=status, **args)
    assert int(status) == 0
    qb = paged_rope(qkv, None, None, ints(past), hq, *b, none, status=status, **args)
    assert int(status) == _lib.DEV_BAD_PAGE and bool(torch.isnan(qb[2 * rows:3 * rows]).all())
    keep = [i for s in (0, 1, 3) for i in table[s].tolist() if i >= 0]
    mine = [i for i in table[2].tolist() if i >= 0]
    for x, y, z in zip(a, b, pool):
        assert torch.equal(bits(y[keep]), bits(x[keep])) and torch.equal(bits(y[mine]), bits(z[mine]))
    other = [r for r in range(4 * rows) if not 2 * rows <= r < 3 * rows]
    assert torch.equal(qa[other], qb[other])


@pytest.mark.parametrize("rows", [1, 3, 40])
def test_positions_out_of_bounds(rows):
    hq, hkv, past = 8, 4, [0, 60, 100]
    table, pages = tables([p + rows for p in past], 9, extra=0)
    pool, _ = pool_of(table, pages, [rows] * 3, past, hkv, False, 10)
    q = normal((3 * rows, hq, 128), 11, rows)
    bound = 100
    out = sq.sq_paged_attention_f16(q, *pool, table, None, ints([-1, 60, 100]), max_rows=rows, len_bound=bound)
    for s, p in enumerate((-1, 60, 100)):
        for j in range(rows):
            assert bool(torch.isnan(out[s * rows + j]).all()) == (not 0 <= p + j < bound), (s, j)
    qkv = normal((3 * rows, (hq + 2 * hkv) * 128), 12, rows).float()
    status = torch.zeros(1, dtype=I32, device=DEV)
    before = [x.clone() for x in pool]
    sq.sq_paged_rope_kv_f16(qkv, None, None, ints([-rows, 2 ** 31 - 1, bound]), hq, *pool, table, max_rows=rows,
                            len_bound=bound, status=status)
    assert int(status) == _lib.DEV_BAD_POS
    for x, y in zip(pool, before):
        assert torch.equal(bits(x), bits(y))


@pytest.mark.parametrize("rows,hq,hkv", [(1, 28, 4), (4, 28, 4), (9, 28, 4), (70, 8, 2)])
@pytest.mark.parametrize("q4", [False, True])
def test_what_the_mask_leaves_out(rows, hq, hkv, q4):
    """Entries behind a row's position do not matter: NaN, infinities and stale ones in the page's rest."""
    paged = calls(q4)[2]
    past = [33, 64, 511]
    table, pages = tables([p + rows for p in past], 13, extra=1)
    pool, (k, v) = pool_of(table, pages, [rows] * 3, past, hkv, q4, 14)
    q = normal((3 * rows, hq, 128), 15, rows)
    args = dict(max_rows=rows)
    good = paged(q, *pool, table, None, ints(past), **args)
    for s, p in enumerate(past):
        end = p + rows
        page, at = int(table[s, end // 64]), end % 64
        if page < 0:
            continue
        if q4:
            pool[0][page, :, at:] = 0xFF
            pool[1][page, :, at:] = float("inf")
            pool[3][page, :, :, at:] = NAN
        else:
            pool[0][page, :, at:] = NAN
            pool[1][page, :, :, at:] = -float("inf")
    assert torch.equal(paged(q, *pool, table, None, ints(past), **args), good)


def test_captured_with_eager_work_between():
    """A graph of write and attention whose table and positions move between replays."""
    hq, hkv, b = 28, 4, 6
    past = [10, 63, 64, 200, 1000, 3000]
    table, pages = tables([p + 4 for p in past], 16)
    pool, _ = pool_of(table, pages, [4] * b, past, hkv, False, 17)
    qkv, pos = normal((b, (hq + 2 * hkv) * 128), 18).float(), ints(past)
    out, q = torch.zeros(b, hq, 128, dtype=F16, device=DEV), torch.zeros(b, hq, 128, dtype=F16, device=DEV)
    tab = table.clone()

    def step(pool, out, q):
        sq.sq_paged_rope_kv_f16(qkv, None, None, pos, hq, *pool, tab, q_out=q, max_rows=1)
        sq.sq_paged_attention_f16(q, *pool, tab, None, pos, out=out, max_rows=1)

    step(pool, out, q)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(pool, out, q)
    for i in range(4):
        twin, o2, q2 = [x.clone() for x in pool], torch.zeros_like(out), torch.zeros_like(q)
        pos.copy_(ints([p + i for p in past]))
        tab.copy_(table[torch.randperm(b, generator=torch.Generator().manual_seed(i)).to(DEV)] if i == 2 else table)
        if i == 2:
            pos.copy_(ints([4] * b))
        step(twin, o2, q2)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, o2) and torch.equal(bits(pool[0]), bits(twin[0])) and torch.equal(bits(pool[1]), bits(twin[1]))


def test_other_stream():
    hq, hkv = 8, 4
    table, pages = tables([500, 900], 19)
    pool, _ = pool_of(table, pages, [1, 1], [499, 899], hkv, False, 20)
    q = normal((2, hq, 128), 21)
    want = sq.sq_paged_attention_f16(q, *pool, table, None, ints([499, 899]), max_rows=1)
    pos = ints([499, 899])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = sq.sq_paged_attention_f16(q, *pool, table, None, pos, max_rows=1)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)
