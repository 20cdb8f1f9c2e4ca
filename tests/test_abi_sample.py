"""Host-side validation of the sampling calls (no GPU: nothing is enqueued on an error)."""
import pytest
import torch

import paper_2609_21704_amd as sq
from paper_2609_21704_amd import _lib

A = 0x7F0000000000
B, C, D, E, F, G, H = (A + (i << 42) for i in range(1, 8))
OK, NULL, SHAPE, ALIGN, ALIAS = 0, 1, 2, 3, 4


def draw(x=A, m=3, v=100, ld=104, t=B, k=C, p=D, mp=E, u=F, token=G, status=None):
    return sq.load().sq_sample_f32(x, m, v, ld, t, k, p, mp, u, token, status, None)


def filt(x=A, m=3, v=100, ld=104, t=B, k=C, p=D, mp=E, out=F, status=None):
    return sq.load().sq_filter_logits_f32(x, m, v, ld, t, k, p, mp, out, status, None)


@pytest.mark.parametrize("call", [draw, filt])
def test_arguments(call):
    for bad in (dict(m=0), dict(m=(1 << 20) + 1), dict(v=0), dict(v=(1 << 26) + 1, ld=1 << 27), dict(ld=99), dict(ld=1 << 31)):
        assert call(**bad) == SHAPE, bad
    assert call(x=None) == NULL and call(x=A + 2) == ALIGN
    for name in ("t", "k", "p", "mp"):
        assert call(**{name: H + 2}) == ALIGN, name
        assert call(**{name: F if call is filt else G}) == ALIAS, name
    assert call(status=H + 1) == ALIGN and call(status=A + 8) == ALIAS and call(status=E + 8) == ALIAS


def test_outputs():
    assert draw(u=None) == NULL and draw(token=None) == NULL and draw(u=F + 1) == ALIGN and draw(token=G + 2) == ALIGN
    assert draw(token=A + 400) == ALIAS and draw(token=F) == ALIAS and draw(token=G, status=G + 8) == ALIAS
    assert filt(out=None) == NULL and filt(out=F + 2) == ALIGN
    # in place is exact; the last logit of the last row
    assert filt(out=A + 4) == ALIAS and filt(out=A + 4 * (2 * 104 + 99)) == ALIAS and filt(out=A, status=A) == ALIAS


def test_binding():
    x, i = torch.zeros(3, 10), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU tensors"):
        sq.sq_sample_f32(x, i)
    with pytest.raises(ValueError, match="logits"):
        sq.sq_sample_f32(x.half(), i)
    with pytest.raises(ValueError, match="logits"):
        sq.sq_filter_logits_f32(x[0])
    for bad in (dict(temperature=i), dict(top_p=i), dict(min_p=i), dict(top_k=x[:, 0].contiguous())):
        with pytest.raises(TypeError):
            sq.sq_sample_f32(x, i, **bad)
    with pytest.raises(ValueError, match="top_k"):
        sq.sq_filter_logits_f32(x, top_k=i[:2])
    assert _lib.DEV_BAD_PARAM == 256
