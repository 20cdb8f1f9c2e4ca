"""GPU checks of the attention over pages of many sequences, whose keys are cut into equal shares (more than 128 / hkv
sequences of few rows): ids outside the pool, entries that the mask leaves out, values that are not finite, idle sequences,
graphs and other streams, with pairs that the borders of shares cut."""
import pytest
import torch

import paper_2609_21704_amd as sq
from paper_2609_21704_amd import _lib
from test_gpu_paged import calls, check_attention, exact, ints, normal, pool_of, starts, tables

pytestmark = pytest.mark.gpu
DEV = "cuda"
NAN, INF = float("nan"), float("inf")
F16 = torch.float16
B, HQ, HKV = 70, 28, 4
# most sequences short, some so long that several borders cut each of their pairs
PAST = [(i * 389) % 1500 if i % 9 else 3000 + 640 * i for i in range(B)]
# rows of a sequence: queries in one tile of 16, in one of 32, in two of 32 (4-bit)
FORMS = [(1, False), (3, False), (4, False), (1, True), (2, True), (9, True)]


def setup(rows, q4, seed, extra=0):
    table, pages = tables([p + rows for p in PAST], seed, extra=extra)
    pool, by_seq = pool_of(table, pages, [rows] * B, PAST, HKV, q4, seed)
    return table, pages, pool, by_seq, normal((B * rows, HQ, 128), seed, rows, std=1.3)


@pytest.mark.parametrize("rows,q4", FORMS)
def test_pages_outside_the_pool(rows, q4):
    """Rows that read a position of no page are NaN, all others have the bits of the call without it."""
    paged = calls(q4)[2]
    table, pages, pool, _, q = setup(rows, q4, 71)
    args = dict(max_rows=rows, len_bound=max(PAST) + rows)
    good = paged(q, *pool, table, None, ints(PAST), **args)
    assert bool(torch.isfinite(good).all())
    bad, first = table.clone(), {}
    for s, place in ((0, 0.5), (9, 0.0), (18, 0.99), (27, 0.3), (63, 0.7), (1, 0.0), (4, 0.99), (69, 0.5)):
        i = int(place * ((PAST[s] + rows + 63) // 64))
        bad[s, i] = (-1, pages, 2 ** 31 - 1, -2 ** 31)[s % 4]
        first[s] = 64 * i
    out = paged(q, *pool, bad, None, ints(PAST), **args)
    for s in range(B):
        for j in range(rows):
            got = out[s * rows + j]
            if PAST[s] + j >= first.get(s, 1 << 30):
                assert bool(torch.isnan(got).all()), (s, j)
            else:
                assert torch.equal(got, good[s * rows + j]), (s, j)


@pytest.mark.parametrize("rows,q4", FORMS)
def test_what_the_mask_leaves_out(rows, q4):
    """NaN, infinities and stale entries behind a row's position do not matter."""
    paged = calls(q4)[2]
    table, _, pool, _, q = setup(rows, q4, 72, extra=1)
    good = paged(q, *pool, table, None, ints(PAST), max_rows=rows)
    assert bool(torch.isfinite(good).all())
    for s, p in enumerate(PAST):
        page, at = int(table[s, (p + rows) // 64]), (p + rows) % 64
        if page < 0:
            continue
        if q4:
            pool[0][page, :, at:], pool[1][page, :, at:], pool[3][page, :, :, at:] = 0xFF, INF, NAN
        else:
            pool[0][page, :, at:], pool[1][page, :, :, at:] = NAN, -INF
    assert torch.equal(paged(q, *pool, table, None, ints(PAST), max_rows=rows), good)


@pytest.mark.parametrize("rows", [1, 4])
def test_values_that_are_not_finite(rows):
    """An infinity or a NaN among the entries that are read reaches those rows, heads and dimensions, as in 64 bits."""
    table, _, pool, (k, v), q = setup(rows, False, 73)
    poison = [(0, 0.0, INF), (9, 0.6, -INF), (18, 1.0, INF), (27, 1.0, NAN), (5, 1.0, -INF), (6, 0.0, NAN), (63, 0.4, INF)]
    for s, place, x in poison:
        key = int(place * PAST[s])
        pool[1][int(table[s, key // 64]), s % HKV, 3 + s, key % 64] = x
        v[s][s % HKV, key, 3 + s] = x
    out = sq.sq_paged_attention_f16(q, *pool, table, None, ints(PAST), max_rows=rows)
    ref = exact(q, k, v, [rows] * B, PAST, [rows * s for s in range(B)])
    odd = ~torch.isfinite(ref)
    assert int(odd.sum()) == sum(rows * HQ // HKV for _ in poison)
    assert torch.equal(torch.isnan(out), torch.isnan(ref)) and torch.equal(out[torch.isinf(ref)].double(), ref[torch.isinf(ref)])
    for s, _, _ in poison:
        v[s][~torch.isfinite(v[s])] = 0
    check_attention(out.masked_fill(odd, 0), ref.masked_fill(odd, 0), v, HQ, True)
    # a key
    pool[0][int(table[36, 2]), 1, 7, 100] = NAN
    out = sq.sq_paged_attention_f16(q, *pool, table, None, ints(PAST), max_rows=rows)
    hit = torch.isnan(out).all(-1).nonzero().tolist()
    assert hit == [[36 * rows + j, h] for j in range(rows) for h in range(HQ // HKV, 2 * HQ // HKV)]


@pytest.mark.parametrize("rows,q4", FORMS)
def test_idle_and_empty_sequences_among_many(rows, q4):
    paged = calls(q4)[2]
    table, _, pool, (k, v), q = setup(rows, q4, 74)
    idle = [s for s in range(B) if s % 5 == 1 or s in (0, 69)]
    lens = [0 if s in (3, 36) else rows for s in range(B)]
    pos = ints([_lib.POS_IDLE if s in idle else p for s, p in enumerate(PAST)])
    start = starts(lens, 2)
    q = normal((sum(lens) + 3, HQ, 128), 75, rows, std=1.3)
    out = torch.full((sum(lens) + 3, HQ, 128), 9.0, dtype=F16, device=DEV)
    paged(q, *pool, table, start, pos, out=out, max_rows=rows)
    first = start.tolist()
    k, v = ([x[:, :n + p] for x, n, p in zip(t, lens, PAST)] for t in (k, v))
    ref = exact(q, k, v, lens, PAST, first)
    live = [r for s in range(B) if s not in idle for r in range(first[s], first[s] + lens[s])]
    rest = [r for r in range(sum(lens) + 3) if r not in live]
    assert bool((out[rest] == 9).all())
    check_attention(out[live], ref[live], v, HQ, not q4)
    # none with rows
    out.fill_(9)
    paged(q, *pool, table, ints([2] * (B + 1)), ints(PAST), out=out, max_rows=rows)
    paged(q, *pool, table, start, ints([_lib.POS_IDLE] * B), out=out, max_rows=rows)
    assert bool((out == 9).all())


@pytest.mark.parametrize("q4", [False, True])
def test_captured_with_eager_work_between(q4):
    """A graph of write and attention whose table and positions move between replays, sequences going idle among them."""
    rope, _, paged, _ = calls(q4)
    table, _, pool, _, _ = setup(4, q4, 76)
    qkv, pos, tab = normal((B, (HQ + 2 * HKV) * 128), 77).float(), ints(PAST), table.clone()
    out, q = (torch.zeros(B, HQ, 128, dtype=F16, device=DEV) for _ in range(2))
    status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def step(pool, out, q):
        rope(qkv, None, None, pos, HQ, *pool, tab, q_out=q, max_rows=1, status=status)
        paged(q, *pool, tab, None, pos, out=out, max_rows=1)

    step(pool, out, q)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(pool, out, q)
    for i in range(5):
        twin, o2, q2 = [x.clone() for x in pool], out.clone(), q.clone()
        if i == 2:
            tab.copy_(table.flip(0))
            pos.copy_(ints([p % 60 for p in PAST]))
        else:
            tab.copy_(table)
            pos.copy_(ints([_lib.POS_IDLE if i == 3 and s % 3 == 0 else p + i % 4 for s, p in enumerate(PAST)]))
        step(twin, o2, q2)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, o2) and torch.equal(q, q2) and int(status) == 0 and bool(torch.isfinite(out).all())
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(pool, twin))


@pytest.mark.parametrize("rows,q4", [(1, False), (9, True)])
def test_other_stream(rows, q4):
    paged = calls(q4)[2]
    table, _, pool, _, q = setup(rows, q4, 78)
    pos = ints(PAST)
    want = paged(q, *pool, table, None, pos, max_rows=rows)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = paged(q, *pool, table, None, pos, max_rows=rows)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
