"""GPU checks of the packed attention at the far ends of its range: positions of millions beside short prompts, scores far
past fp32's whole numbers, weights to more than binary16, split keys of many sequences, prompts packed beside single tokens."""
import math

import pytest
import torch

import paper_2609_21704_amd as sq
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
