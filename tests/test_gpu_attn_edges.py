"""Attention over the paged cache where it can go wrong: how exact 16-bit results are, lengths beyond the table, lists that do not rise, NaN over whole runs."""
import math

import pytest
import torch

from paper_2602_06694_amd import binding as nq
from decoder_util import NQ, TORCH, attention, close, randn
from test_gpu_attn import Problem, random_tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new,ctx", [(1, 4000), (4, 1500), (9, 900), (16, 2000)])
def test_16_bit_results_of_few_rows_are_rounded_once(dtype, d, new, ctx):
    """The distance from binary64 in the 2-norm is that of binary64 results rounded to the type.  Weights of 16 bits and more are off by 2^-17 at most, scores of some 10 by
    2^-20 of a weight: below a hundredth of the rounding's root mean square (0.4 half units of 2^-9 in bf16; of 2^-12 in fp16, whose weights have 22 bits)."""
    p = Problem(51 + d, [ctx], [new], 4, 1, d, dtype, dtype, tree=[random_tree(new, 4)])
    got, _ = p.run()
    want, _ = attention(p.q.double().view(new, 4, d), p.k[0].double(), p.v[0].double(), p.see(0), p.scale)
    once = float((want.to(TORCH[dtype]).double() - want).norm())
    assert float((got.double() - want).norm()) <= 1.02 * once
    p.done()
