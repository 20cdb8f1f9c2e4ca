"""Host-side validation of the calls over packed rows and the 4-bit cache (no GPU: nothing is enqueued on an error)."""
import pytest
import torch

import paper_2609_21704_amd as sq
from paper_2609_21704_amd import _lib

A = 0x7F0000000000
B, C, D, E, F, G, H, I = (A + (i << 36) for i in range(1, 9))
OK, NULL, SHAPE, ALIGN, ALIAS, NONFINITE = 0, 1, 2, 3, 4, 5


def rope_f16(qkv=A, bias=None, start=B, b=2, rows=10, most=8, hq=4, hkv=2, pos=C, lb=128, cap=128, theta=1e6, q=D, k=E,
             v=F, status=None):
    return sq.load().sq_packed_rope_kv_f16(qkv, bias, start, b, rows, most, hq, hkv, pos, 0, lb, cap, theta, q, k, v,
                                           status, None)


def rope_q4(q=D, kc=E, ks=F, vc=G, vs=H, cap=128, status=None, start=B):
    return sq.load().sq_packed_rope_kv_q4(A, None, start, 2, 10, 8, 4, 2, C, 0, 128, cap, 1e6, q, kc, ks, vc, vs, status,
                                          None)


def read_q4(kc=E, ks=F, vc=G, vs=H, rows=10, ko=D, vo=I):
    return sq.load().sq_packed_kv_read_q4(kc, ks, vc, vs, B, 2, rows, 8, 2, C, 0, 128, 128, ko, vo, None)


def attn_f16(q=A, k=E, v=F, start=B, b=2, rows=10, most=8, hq=4, hkv=2, pos=C, lb=128, cap=128, out=D):
    return sq.load().sq_packed_attention_f16(q, k, v, start, b, rows, most, hq, hkv, pos, 0, lb, cap, out, None)


def attn_q4(kc=E, ks=F, vc=G, vs=H, out=D):
    return sq.load().sq_packed_attention_q4(A, kc, ks, vc, vs, B, 2, 10, 8, 4, 2, C, 0, 128, 128, out, None)


@pytest.mark.parametrize("call", [rope_f16, attn_f16])
@pytest.mark.parametrize("bad", [dict(b=0), dict(rows=-1), dict(rows=(1 << 20) + 1), dict(most=0), dict(most=(1 << 20) + 1),
                                 dict(hq=5), dict(hkv=0), dict(hq=130, hkv=1), dict(cap=100, lb=100), dict(lb=129),
                                 dict(lb=0), dict(b=40000, hkv=2), dict(start=None), dict(start=None, b=2, rows=17)])
def test_sizes(call, bad):
    assert call(**bad) == SHAPE


def test_capacity():
    big = (1 << 28) + 64
    assert attn_f16(cap=big) == SHAPE and attn_f16(cap=big, rows=0) == SHAPE and rope_f16(cap=big, rows=0) == OK
    assert attn_f16(cap=1 << 28, rows=0) == OK


def test_pointers():
    assert rope_f16(qkv=None) == NULL and rope_f16(pos=None) == NULL and rope_f16(k=None) == NULL
    assert rope_f16(q=None) == NULL and rope_f16(theta=float("inf")) == NONFINITE and rope_f16(theta=1.0) == SHAPE
    assert rope_f16(qkv=A + 4) == ALIGN and rope_f16(start=B + 2) == ALIGN and rope_f16(status=I + 1) == ALIGN
    assert rope_f16(bias=I + 8) == ALIGN
    assert rope_f16(q=A + 16) == ALIAS and rope_f16(k=F) == ALIAS and rope_f16(status=C) == ALIAS
    assert rope_f16(start=D + 64) == ALIAS
    for name in ("kc", "ks", "vc", "vs"):
        for call in (rope_q4, read_q4, attn_q4):
            assert call(**{name: None}) == NULL, (name, call)
            assert call(**{name: E + 8}) == ALIGN, (name, call)
    assert rope_q4(vs=G + 64) == ALIAS and rope_q4(status=H) == ALIAS
    assert read_q4(ko=None) == NULL and read_q4(vo=D + 16) == ALIAS and read_q4(ko=G) == ALIAS
    assert attn_f16(out=None) == NULL and attn_f16(out=D + 8) == ALIGN and attn_f16(out=A) == ALIAS
    assert attn_f16(out=F + 256) == ALIAS and attn_f16(out=B) == ALIAS and attn_q4(out=H) == ALIAS


def test_no_rows():
    assert rope_f16(rows=0, qkv=None, q=None) == OK and attn_f16(rows=0, q=None, out=None) == OK
    assert read_q4(rows=0, ko=None) == OK and rope_f16(rows=0, most=0) == SHAPE


def test_binding():
    u8, f16, i32 = torch.uint8, torch.float16, torch.int32
    cache = (torch.zeros(2, 1, 64, 64, dtype=u8), torch.zeros(2, 1, 64, 4, dtype=f16),
             torch.zeros(2, 1, 1, 64, 64, dtype=u8), torch.zeros(2, 1, 1, 4, 64, dtype=f16))
    q, start, pos = torch.zeros(5, 2, 128, dtype=f16), torch.zeros(3, dtype=i32), torch.zeros(2, dtype=i32)
    with pytest.raises(ValueError, match="GPU tensors"):
        sq.sq_packed_attention_q4(q, *cache, start, pos)
    with pytest.raises(ValueError, match="row_start"):
        sq.sq_packed_attention_q4(q, *cache, start[:2], pos)
    with pytest.raises(ValueError, match="same number"):
        sq.sq_packed_attention_q4(q, *cache, None, pos)
    with pytest.raises(TypeError, match="pos_base"):
        sq.sq_packed_attention_q4(q, *cache, start, pos.long())
    with pytest.raises(ValueError, match="v_scales"):
        sq.sq_packed_attention_q4(q, *cache[:3], cache[1], start, pos)
    with pytest.raises(ValueError, match="multiple of 64"):
        sq.sq_packed_kv_read_q4(cache[0][:, :, :32], *cache[1:], start, pos, 5)
    with pytest.raises(ValueError, match="float16"):
        sq.sq_packed_attention_q4(q.float(), *cache, start, pos)
    with pytest.raises(ValueError, match="qkv"):
        sq.sq_packed_rope_kv_q4(torch.zeros(5, 100), None, start, pos, 2, *cache)
    assert _lib.DEV_BAD_ROWS == 16
