"""GPU checks of the sampling calls (include/specquant_sample.h) against the definition in 64 bits and whole numbers: every
filter alone and together, ties, masked and invalid rows, the ends of the settings, odd vocabularies, padded rows."""
import math

import numpy as np
import pytest
import torch

import paper_2609_21704_amd as sq
from paper_2609_21704_amd import _lib

pytestmark = pytest.mark.gpu
DEV = "cuda"
INF, NAN = float("inf"), float("nan")


def kept(x, temp, k, p, mp):
    """(weights on the grid, kept) of a row, None where it has no distribution or a bad setting."""
    x = np.asarray(x, np.float32)
    v = x.size
    if not (0 <= temp < INF) or not p >= 0 or not mp >= 0 or np.isnan(x).any() or (x == INF).any() or (x == -INF).all():
        return None
    x = x.astype(np.float64)
    if temp == 0:
        keep = np.arange(v) == int(np.argmax(x))
        return keep.astype(np.int64), keep
    z = x / np.float64(np.float32(temp))
    w = np.exp(z - z.max()).astype(np.float32)
    r = np.rint(w.astype(np.float64) * 2.0 ** min(51, 62 - (v - 1).bit_length())).astype(np.int64)
    order = np.lexsort((np.arange(v), -x))
    if 0 < k < v:
        order = order[:k]
    if p < 1:
        run = np.cumsum(r[order])
        need = max(1, math.ceil(float(np.float32(p)) * float(int(run[-1]))))
        order = order[:int(np.searchsorted(run - r[order], need))]
    keep = np.zeros(v, bool)
    keep[order] = True
    return r, keep & (w >= np.float32(min(mp, 1.0)))


def token(x, u24, *setting):
    rk = kept(x, *setting)
    if rk is None:
        return -1
    ids = rk[1].nonzero()[0]
    run = np.cumsum(rk[0][ids])
    return int(ids[np.searchsorted(run, ((u24 & 0xFFFFFF) * int(run[-1])) >> 24, side="right")])


def device(settings):
    t, k, p, mp = zip(*settings)
    f = dict(dtype=torch.float32, device=DEV)
    return dict(temperature=torch.tensor(t, **f), top_k=torch.tensor(k, dtype=torch.int32, device=DEV),
                top_p=torch.tensor(p, **f), min_p=torch.tensor(mp, **f))


def check(logits, settings, vocab=None, seed=0, draws=3):
    """Filtered logits and tokens of every row; logits: a float32 tensor [m][ld] on the host."""
    v = vocab or logits.shape[1]
    g = torch.Generator().manual_seed(seed)
    x, d = logits.to(DEV), device(settings)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = sq.sq_filter_logits_f32(x, vocab=v, out=torch.full_like(x, 5.0), status=status, **d).cpu()
    want, bits = torch.full_like(logits, 5.0), 0
    for i, s in enumerate(settings):
        row = logits[i, :v].numpy()
        rk = kept(row, *s)
        if rk is None:
            bad = not (0 <= s[0] < INF) or not s[2] >= 0 or not s[3] >= 0
            bits |= _lib.DEV_BAD_PARAM if bad else 8
            want[i, :v] = NAN if bad else torch.from_numpy(row)
        else:
            want[i, :v] = torch.from_numpy(np.where(rk[1], row, -np.float32(INF)))
    assert torch.equal(torch.nan_to_num(out, nan=7e7), torch.nan_to_num(want, nan=7e7)), \
        [(i, settings[i], int((out[i] != want[i]).sum())) for i in range(len(settings)) if not torch.equal(out[i], want[i])][:4]
    assert int(status) == bits
    same = x.clone()
    sq.sq_filter_logits_f32(same, vocab=v, out=same, **d)
    assert torch.equal(torch.nan_to_num(same[:, :v].cpu(), nan=7e7), torch.nan_to_num(want[:, :v], nan=7e7))
    for n in range(draws):
        u = torch.randint(-2 ** 31, 2 ** 31, (len(settings),), generator=g, dtype=torch.int32)
        if n == 0:
            u[::2], u[1::2] = 0, 0xFFFFFF
        got = sq.sq_sample_f32(x, u.to(DEV), vocab=v, **d).tolist()
        assert got == [token(logits[i, :v].numpy(), int(u[i]), *s) for i, s in enumerate(settings)]


SETTINGS = [(1.0, 0, 1.0, 0.0), (0.7, 5, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (1.2, 0, 1.0, 0.05), (0.8, 50, 0.95, 0.0),
            (1.0, 40, 0.5, 0.1), (2.0, 1, 0.3, 0.0), (0.0, 3, 0.1, 0.5), (1.0, 10 ** 9, 0.999, 0.0), (3.0, 7, 2.0, 9.0),
            (1.0, 0, 0.0, 0.0), (0.1, 100, 0.99999, 1e-30), (1.0, -5, 1.0, 1.0), (50.0, 300, 0.8, 0.9)]


@pytest.mark.parametrize("v", [1, 2, 3, 63, 64, 65, 1000, 4096, 4097, 32000, 151936])
@pytest.mark.parametrize("std", [0.5, 4.0])
def test_filters(v, std):
    g = torch.Generator().manual_seed(v)
    check(torch.randn(len(SETTINGS), v, generator=g) * std, SETTINGS)


@pytest.mark.parametrize("m,v,ld", [(1, 151936, 151936), (1, 5000, 5003), (17, 20001, 20032), (70, 9000, 9000), (300, 700, 701),
                                    (1100, 50, 53)])
def test_rows(m, v, ld):
    """From one row to more than fit the scratch at once; rows longer than the vocabulary."""
    g = torch.Generator().manual_seed(m)
    x = torch.randn(m, ld, generator=g) * 3
    x[:, v:] = 100.0
    check(x, [SETTINGS[i % len(SETTINGS)] for i in range(m)], vocab=v, seed=1)


@pytest.mark.parametrize("v", [70, 5000, 30000])
def test_ties(v):
    """Equal logits at the cuts, and more of them than are ranked against each other: the lowest index goes first."""
    g = torch.Generator().manual_seed(v)
    rows = [torch.zeros(v), torch.full((v,), -3.25), torch.randint(-2, 3, (v,), generator=g).float(),
            torch.randint(-40, 41, (v,), generator=g).float() / 8, torch.randn(v, generator=g).half().float(),
            torch.where(torch.rand(v, generator=g) < 0.5, 0.0, -0.0), torch.randn(v, generator=g) * 1e-6 + 10]
    rows[-1][5] = -1e30  # far below: the others share a bin
    x = torch.stack([r for r in rows for _ in SETTINGS])
    check(x, SETTINGS * len(rows))


@pytest.mark.parametrize("n", [1, 63, 64, 65, 95, 96, 97, 130, 511, 512, 513])
@pytest.mark.parametrize("step", [0.0, 2.0 ** -22])
def test_crowded(n, step):
    """Cuts at the ends of and inside a group of n tokens that no bins tell apart, up to more than are ranked."""
    g = torch.Generator().manual_seed(n)
    v = 3000
    x = torch.randn(v, generator=g) * 4
    order = torch.randperm(v, generator=g)[:n]
    x[order] = 2.0 + step * torch.randint(0, 9, (n,), generator=g)
    above = int((x > 3.0).sum())
    cuts = sorted({above + i for i in (1, n // 3 + 1, n - 1, n, n + 1)} | {max(above, 1)})
    full = torch.softmax(x.double(), 0)
    mass, group = float(full[x > 3.0].sum()), float(full[order].sum())
    settings = [(1.0, k, 1.0, 0.0) for k in cuts if k > 0] + [(1.0, 0, mass + p * group, 0.0) for p in (0.01, 0.5, 0.99)] \
        + [(1.0, above + n // 2 + 1, p, 0.0) for p in (0.5, 0.9, 0.999)]
    check(x.repeat(len(settings), 1), settings)


def test_large():
    """A vocabulary of millions, and rows that lie more than 2^31 logits apart."""
    g = torch.Generator().manual_seed(21)
    v = (1 << 22) + 3
    check(torch.randn(3, v, generator=g) * 2, [(0.9, 1000, 0.9, 0.0), (1.0, 0, 0.99, 0.0), (1.3, 0, 1.0, 0.01)], draws=2)
    x, far = torch.randn(4, 999, generator=g), torch.empty(4, 1 << 30, device=DEV)
    far[:, :999] = x.to(DEV)
    settings = [(0.8, 50, 0.95, 0.0), (1.0, 0, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 20, 1.0, 0.1)]
    u = torch.randint(0, 1 << 24, (4,), generator=g, dtype=torch.int32)
    got = sq.sq_sample_f32(far, u.to(DEV), vocab=999, **device(settings)).tolist()
    assert got == [token(x[i].numpy(), int(u[i]), *s) for i, s in enumerate(settings)]
    sq.sq_filter_logits_f32(far, vocab=999, out=far, **device(settings))
    want = sq.sq_filter_logits_f32(x.to(DEV), **device(settings))
    assert torch.equal(far[:, :999], want)


def test_far_apart():
    """Logits at the ends of fp32, and temperatures that take their quotients there."""
    v = 3000
    g = torch.Generator().manual_seed(5)
    big, tiny = 3.4e38, 1e-42
    rows = [torch.randn(v, generator=g) * 1e38, torch.full((v,), big), torch.randn(v, generator=g) * tiny,
            torch.cat([torch.full((1,), big), torch.full((v - 1,), -big)]), torch.linspace(-30, 30, v)]
    settings = [(t, k, p, mp) for t in (1e-38, 1.0, 3e38) for k, p, mp in ((0, 0.9, 0.0), (7, 1.0, 0.0), (0, 1.0, 0.3), (9, 0.6, 0.1))]
    x = torch.stack([r.clamp(-big, big) for r in rows for _ in settings])
    check(x, settings * len(rows))


def test_masked_and_invalid():
    v = 6000
    g = torch.Generator().manual_seed(6)
    rows = [torch.randn(v, generator=g) * 2 for _ in range(6)]
    rows[0][torch.rand(v, generator=g) < 0.7] = -INF
    rows[1][:] = -INF
    rows[1][4321] = -7.0        # one token is left
    rows[2][:] = -INF           # none is
    rows[3][17] = NAN
    rows[4][v - 1] = INF
    rows[5][3:] = -INF          # fewer than top-k keeps
    x = torch.stack([r for r in rows for _ in SETTINGS])
    check(x, SETTINGS * len(rows))
    bad = [(NAN, 0, 1.0, 0.0), (-1.0, 0, 0.9, 0.0), (INF, 5, 1.0, 0.0), (1.0, 5, NAN, 0.0), (1.0, 0, -0.1, 0.0), (1.0, 0, 0.9, NAN),
           (0.0, 0, 1.0, -1.0), (1.0, 0, 0.5, 0.0)]
    check(torch.randn(len(bad), v, generator=g), bad)


def test_every_draw_of_a_small_row():
    """All 2^24 numbers would draw each token as often as its weight says: here every 4099th."""
    x = torch.tensor([[0.3, -1.0, 2.0, -INF, 0.3, -20.0, 1.5]])
    u = torch.arange(0, 1 << 24, 4099, dtype=torch.int32)
    rows = x.expand(u.numel(), -1).contiguous()
    for s in ((1.0, 0, 1.0, 0.0), (1.5, 4, 0.9, 0.0)):
        d = device([s] * u.numel())
        got = sq.sq_sample_f32(rows.to(DEV), u.to(DEV), **d).cpu().numpy()
        r, keep = kept(x[0].numpy(), *s)
        share = np.where(keep, r, 0) / r[keep].sum()
        count = np.bincount(got, minlength=7) / u.numel()
        assert np.abs(count - share).max() <= 2 / u.numel()  # (a border in a step at each end)


def test_without_settings():
    """Arrays left out: temperature 1 and no filter, which is sq_spec_accept's draw but for borders 2^-23 apart."""
    g = torch.Generator().manual_seed(8)
    x = (torch.randn(40, 32000, generator=g) * 2).to(DEV)
    u = torch.randint(0, 1 << 24, (40,), generator=g, dtype=torch.int32).to(DEV)
    got = sq.sq_sample_f32(x, u)
    n, want = sq.sq_spec_accept(None, x.view(40, 1, -1), None, u.view(40, 1), 1.0)[:2]
    assert int((got != want).sum()) == 0
    assert torch.equal(sq.sq_filter_logits_f32(x), x)
    k = torch.full((40,), 3, dtype=torch.int32, device=DEV)
    assert int((sq.sq_filter_logits_f32(x, top_k=k) > -INF).sum()) == 120
    assert torch.equal(sq.sq_sample_f32(x, u, top_k=k.fill_(1)).long(), x.argmax(-1))


def test_captured():
    """A graph of filter and draw whose logits and settings move between replays, with eager calls between."""
    m, v = 9, 33000
    g = torch.Generator().manual_seed(9)
    x, out = torch.zeros(m, v, device=DEV), torch.zeros(m, v, device=DEV)
    u, tok = torch.zeros(m, dtype=torch.int32, device=DEV), torch.zeros(m, dtype=torch.int32, device=DEV)
    d = device(SETTINGS[:m])

    def step():
        sq.sq_filter_logits_f32(x, out=out, **d)
        sq.sq_sample_f32(x, u, token=tok, **d)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        rows, un = torch.randn(m, v, generator=g) * (1 + i), torch.randint(0, 1 << 24, (m,), generator=g, dtype=torch.int32)
        settings = SETTINGS[i:i + m]
        x.copy_(rows)
        u.copy_(un)
        for k, t in device(settings).items():
            d[k].copy_(t)
        want = sq.sq_filter_logits_f32(x, **d)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert tok.tolist() == [token(rows[j].numpy(), int(un[j]), *s) for j, s in enumerate(settings)]
