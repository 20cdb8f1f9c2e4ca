"""Host-side validation of the calls over paged caches (no GPU: nothing is enqueued on an error)."""
import pytest
import torch

import paper_2609_21704_amd as sq
from paper_2609_21704_amd import _lib

A = 0x7F0000000000
B, C, D, E, F, G, H, I, J = (A + (i << 36) for i in range(1, 10))
OK, NULL, SHAPE, ALIGN, ALIAS, NONFINITE = 0, 1, 2, 3, 4, 5


def reserve(table=A, held=B, refs=C, b=4, width=8, pages=20, pos=D, ahead=1, status=None):
    return sq.load().sq_pages_reserve(table, held, refs, b, width, pages, pos, ahead, status, None)


def trim(table=A, held=B, refs=C, b=4, width=8, pages=20, pos=D, status=None):
    return sq.load().sq_pages_trim(table, held, refs, b, width, pages, pos, status, None)


def fork(table=A, held=B, refs=C, b=4, width=8, pages=20, parent=D, child=E, length=F, n=3, src=G, dst=H, count=I,
         status=None):
    return sq.load().sq_pages_fork(table, held, refs, b, width, pages, parent, child, length, n, src, dst, count, status,
                                   None)


def compact(table=A, held=B, refs=C, b=4, width=8, pages=20, src=D, dst=E, count=F, used=G, status=None):
    return sq.load().sq_pages_compact(table, held, refs, b, width, pages, src, dst, count, used, status, None)


def copy(pool=A, layers=2, pages=20, page_bytes=4096, src=B, dst=C, count=D, n=5, status=None):
    return sq.load().sq_page_copy(pool, layers, pages, page_bytes, src, dst, count, n, status, None)


def rope_f16(qkv=A, bias=None, start=B, b=2, rows=10, most=8, hq=4, hkv=2, pos=C, lb=128, table=G, width=2, pages=9,
             theta=1e6, q=D, k=E, v=F, status=None):
    return sq.load().sq_paged_rope_kv_f16(qkv, bias, start, b, rows, most, hq, hkv, pos, 0, lb, table, width, pages, theta,
                                          q, k, v, status, None)


def rope_q4(q=D, kc=E, ks=F, vc=G, vs=H, status=None, table=J):
    return sq.load().sq_paged_rope_kv_q4(A, None, B, 2, 10, 8, 4, 2, C, 0, 128, table, 2, 9, 1e6, q, kc, ks, vc, vs, status,
                                         None)


def read_q4(kc=E, ks=F, vc=G, vs=H, rows=10, ko=D, vo=I, table=J):
    return sq.load().sq_paged_kv_read_q4(kc, ks, vc, vs, table, 2, 9, B, 2, rows, 8, 2, C, 0, 128, ko, vo, None)


def attn_f16(q=A, k=E, v=F, start=B, b=2, rows=10, most=8, hq=4, hkv=2, pos=C, lb=128, table=G, width=2, pages=9, out=D):
    return sq.load().sq_paged_attention_f16(q, k, v, table, width, pages, start, b, rows, most, hq, hkv, pos, 0, lb, out,
                                            None)


def attn_q4(kc=E, ks=F, vc=G, vs=H, out=D, table=J):
    return sq.load().sq_paged_attention_q4(A, kc, ks, vc, vs, table, 2, 9, B, 2, 10, 8, 4, 2, C, 0, 128, out, None)


@pytest.mark.parametrize("call", [reserve, trim, fork, compact])
def test_state(call):
    for bad in (dict(b=0), dict(b=65536), dict(width=0), dict(width=(1 << 20) + 1), dict(pages=0),
                dict(pages=(1 << 20) + 1)):
        assert call(**bad) == SHAPE, bad
    for name in ("table", "held", "refs"):
        assert call(**{name: None}) == NULL and call(**{name: J + 2}) == ALIGN, name
    assert call(held=A) == ALIAS and call(refs=A + 64) == ALIAS and call(status=C + 4) == ALIAS and call(status=J + 1) == ALIGN


def test_state_arguments():
    assert reserve(pos=None) == NULL and reserve(pos=D + 1) == ALIGN and reserve(pos=A + 4) == ALIAS
    assert reserve(ahead=-1) == SHAPE and reserve(ahead=(1 << 20) + 1) == SHAPE
    assert trim(pos=None) == NULL and trim(pos=C) == ALIAS
    assert fork(n=-1) == SHAPE and fork(n=1025) == SHAPE and fork(count=None) == NULL
    for name in ("parent", "child", "length", "src", "dst"):
        assert fork(**{name: None}) == NULL and fork(**{name: J + 2}) == ALIGN, name
    assert fork(src=D) == ALIAS and fork(dst=G + 8) == ALIAS and fork(count=F + 8) == ALIAS and fork(parent=B) == ALIAS
    for name in ("src", "dst", "count", "used"):
        assert compact(**{name: None}) == NULL and compact(**{name: J + 2}) == ALIGN, name
    assert compact(src=B) == ALIAS and compact(dst=D + 36) == ALIAS and compact(used=F) == ALIAS


def test_copy():
    for bad in (dict(layers=0), dict(layers=65536), dict(pages=0), dict(pages=(1 << 20) + 1), dict(page_bytes=8),
                dict(page_bytes=24), dict(page_bytes=(1 << 30) + 16), dict(n=-1), dict(n=(1 << 20) + 1),
                dict(pages=1 << 20, layers=65535, page_bytes=1 << 20)):
        assert copy(**bad) == SHAPE, bad
    assert copy(n=0, pool=None, src=None) == OK
    for name in ("pool", "src", "dst", "count"):
        assert copy(**{name: None}) == NULL and copy(**{name: J + 2}) == ALIGN, name
    assert copy(src=A + 4096) == ALIAS and copy(count=A) == ALIAS and copy(status=B + 4) == ALIAS
    assert copy(src=A + 2 * 20 * 4096 - 4) == ALIAS


@pytest.mark.parametrize("call", [rope_f16, attn_f16])
@pytest.mark.parametrize("bad", [dict(b=0), dict(rows=-1), dict(rows=(1 << 20) + 1), dict(most=0), dict(most=(1 << 20) + 1),
                                 dict(hq=5), dict(hkv=0), dict(hq=130, hkv=1), dict(width=0), dict(width=(1 << 20) + 1),
                                 dict(lb=129), dict(lb=0), dict(b=40000, hkv=2), dict(start=None), dict(pages=0),
                                 dict(pages=(1 << 20) + 1), dict(start=None, b=2, rows=17)])
def test_sizes(call, bad):
    assert call(**bad) == SHAPE


def test_pointers():
    assert rope_f16(qkv=None) == NULL and rope_f16(pos=None) == NULL and rope_f16(k=None) == NULL
    assert rope_f16(q=None) == NULL and rope_f16(theta=float("inf")) == NONFINITE and rope_f16(theta=1.0) == SHAPE
    assert rope_f16(qkv=A + 4) == ALIGN and rope_f16(start=B + 2) == ALIGN and rope_f16(status=I + 1) == ALIGN
    assert rope_f16(q=A + 16) == ALIAS and rope_f16(k=F) == ALIAS and rope_f16(status=C) == ALIAS
    assert rope_f16(table=None) == NULL and rope_f16(table=G + 2) == ALIGN and rope_f16(table=E + 64) == ALIAS
    for name in ("kc", "ks", "vc", "vs"):
        for call in (rope_q4, read_q4, attn_q4):
            assert call(**{name: None}) == NULL, (name, call)
            assert call(**{name: E + 8}) == ALIGN, (name, call)
    assert rope_q4(vs=G + 64) == ALIAS and rope_q4(status=H) == ALIAS and rope_q4(table=H) == ALIAS
    assert read_q4(ko=None) == NULL and read_q4(vo=D + 16) == ALIAS and read_q4(ko=G) == ALIAS and read_q4(table=D) == ALIAS
    assert attn_f16(out=None) == NULL and attn_f16(out=D + 8) == ALIGN and attn_f16(out=A) == ALIAS
    assert attn_f16(out=F + 256) == ALIAS and attn_f16(out=B) == ALIAS and attn_q4(out=H) == ALIAS
    assert attn_f16(table=None) == NULL and attn_f16(table=D) == ALIAS
    # the pool's last byte, which is past what two sequences of 128 positions would take
    assert attn_f16(out=E + 9 * 2 * 64 * 256 - 16) == ALIAS


def test_no_rows():
    assert rope_f16(rows=0, qkv=None, q=None) == OK and attn_f16(rows=0, q=None, out=None) == OK
    assert read_q4(rows=0, ko=None) == OK and rope_f16(rows=0, most=0) == SHAPE


def test_binding():
    i32, f16 = torch.int32, torch.float16
    table, held, refs, pos = (torch.zeros(s, dtype=i32) for s in ((2, 3), (2,), (8,), (2,)))
    k, v, q = torch.zeros(8, 1, 64, 128, dtype=f16), torch.zeros(8, 1, 128, 64, dtype=f16), torch.zeros(2, 2, 128, dtype=f16)
    with pytest.raises(ValueError, match="GPU tensors"):
        sq.sq_pages_reserve(table, held, refs, pos)
    with pytest.raises(ValueError, match="GPU tensors"):
        sq.sq_paged_attention_f16(q, k, v, table, None, pos)
    with pytest.raises(ValueError, match="table"):
        sq.sq_pages_trim(table.long(), held, refs, pos)
    with pytest.raises(ValueError, match="table"):
        sq.sq_paged_attention_f16(q, k, v, table[0], None, pos)
    with pytest.raises(ValueError, match="held"):
        sq.sq_pages_trim(table, held[:1], refs, pos)
    with pytest.raises(ValueError, match="v_pages"):
        sq.sq_paged_attention_f16(q, k, k, table, None, pos)
    with pytest.raises(ValueError, match="src"):
        sq.sq_pages_compact(table, held, refs, pos, torch.zeros(4, dtype=i32), held, held)
    with pytest.raises(ValueError, match="dst"):
        sq.sq_pages_fork(table, held, refs, pos, pos, pos, pos, held[:1], held)
    with pytest.raises(ValueError, match="layers"):
        sq.sq_page_copy(k[0, 0], pos, pos, held)
    with pytest.raises(ValueError, match="k_codes"):
        sq.sq_paged_attention_q4(q, k[0], k, k, k, table, None, pos)
    assert (_lib.DEV_NO_PAGES, _lib.DEV_BAD_PAGE, _lib.DEV_BAD_FORK, _lib.PAGE) == (32, 64, 128, 64)
