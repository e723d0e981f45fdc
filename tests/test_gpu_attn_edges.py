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


@pytest.mark.parametrize("begin,ctx,tokens,hq,hk", [([0, 2048] * 5, [30000] * 9, 2048, 8, 8), ([0, 320] * 7, [64] * 12 + [60000], 320, 64, 8),
                                                    ([0, 17] * 20, [5000] * 39, 17, 8, 1)])
def test_lists_that_do_not_rise_leave_what_is_behind_the_workspace(begin, ctx, tokens, hq, hk):
    """More tiles than rows: what has no place in the workspace is left out.  All sequences in one page, 64 MiB of a pattern behind the workspace."""
    d, page = 128, 16
    begin = begin[:len(ctx) + 1]
    k, v = (randn(i, 1, hk, page, d).to(torch.bfloat16).cuda() for i in (1, 2))
    kv = nq.nq_kv_create(k, v, nq.NQ_BF16, hk, d, page, 1)
    a = nq.nq_attn_create(kv, hq, 0.1, 0.0, nq.NQ_BF16)
    need = nq.nq_attn_workspace_bytes(a, len(ctx), tokens)
    room = torch.full((need + (64 << 20),), 0x5a, dtype=torch.uint8, device="cuda")
    on = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    q, out = randn(3, tokens, hq * d).to(torch.bfloat16).cuda(), torch.zeros(tokens, hq * d, dtype=torch.bfloat16, device="cuda")
    table = torch.zeros(len(ctx), (max(ctx) + tokens) // page + 1, dtype=torch.int32, device="cuda")
    nq.nq_attn_forward(a, q, on(begin), on(ctx), table, None, out, None, room, need)
    torch.cuda.synchronize()
    assert bool((room[need:] == 0x5a).all())
    nq.nq_attn_destroy(a)
    nq.nq_kv_destroy(kv)


def beyond_the_table(new, ctx, pages, tree=None, d=64, hq=4, page=16):
    """One sequence of more tokens than its table has room for: all rows see what the table holds, once."""
    k, v = (randn(70 + i, pages * page, 1, d).to(torch.bfloat16) for i in (1, 2))
    kc, vc = (t.view(pages, page, 1, d).transpose(1, 2).contiguous().cuda() for t in (k, v))
    kv = nq.nq_kv_create(kc, vc, nq.NQ_BF16, 1, d, page, pages)
    a = nq.nq_attn_create(kv, hq, 0.125, 0.0, nq.NQ_F32)
    n = nq.nq_attn_workspace_bytes(a, 1, new)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    on = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    q, out, lse = randn(73, new, hq * d).to(torch.bfloat16), torch.empty(new, hq * d, device="cuda"), torch.empty(new, hq, device="cuda")
    nq.nq_attn_forward(a, q.cuda(), on([0, new]), on([ctx]), on([list(range(pages))]), tree, out, lse, ws, n)
    torch.cuda.synchronize()
    nq.nq_attn_destroy(a)
    nq.nq_kv_destroy(kv)
    want, want_lse = attention(q.double().view(new, hq, d), k.double(), v.double(), torch.ones(new, pages * page, dtype=torch.bool), 0.125)
    # (scores of at most some 20: a weight is off by 2^-17 of itself at most, values are below 5)
    close(out.view(new, hq, d), want, "f32", 2.0 ** -14)
    close(lse, want_lse, "f32", 2.0 ** -16)


@pytest.mark.parametrize("with_tree", [False, True])
@pytest.mark.parametrize("new", [10, 40])
def test_lengths_near_the_end_of_32_bits(new, with_tree):
    """Tiles of 64 and of 128 rows."""
    beyond_the_table(new, 2 ** 31 - 1, 5, torch.zeros(new, 2, dtype=torch.int32, device="cuda") if with_tree else None)


@pytest.mark.parametrize("new", [1, 3, 10, 40])
@pytest.mark.parametrize("pages", [1, 3, 5, 6])
@pytest.mark.parametrize("more", [0, 1, 15, 16, 17, 1000, 2 ** 30])
def test_tokens_beyond_the_table_are_not_seen(new, pages, more):
    """Tables of an odd number of pages of 16 end in the middle of a step of 32 keys."""
    beyond_the_table(new, 16 * pages + more, pages)


NAN_CASES = [([4000], [1], 4, 2, 128), ([9000], [3], 8, 1, 64), ([5000], [20], 4, 1, 128), ([4000], [45], 16, 2, 64), ([3000] * 40, [1] * 40, 16, 2, 64), ([6000, 10], [9, 1], 4, 2, 256)]


def nan_problem(ctx, new, hq, hk, d):
    """Calls whose rows are cut into runs: a row or more to a workgroup of the join, tiles of 16, 64 and 128."""
    return Problem(81, ctx, new, hq, hk, d, "bf16", "f32", tree=[random_tree(n, 6) for n in new])


@pytest.mark.parametrize("case", NAN_CASES)
def test_a_query_of_nan_gives_nan(case):
    ctx, new, hq, hk, d = case
    p = nan_problem(*case)
    clean, clean_lse = p.run()
    p.q[0, d:2 * d], p.q[-1, 0] = math.nan, math.nan             # all of a head, one element of another
    out, lse = p.run()
    bad = torch.zeros(sum(new), hq, dtype=torch.bool)
    bad[0, 1] = bad[-1, 0] = True
    assert bool(torch.isnan(out[bad]).all()) and bool(torch.isnan(lse[bad]).all())
    assert torch.equal(out[~bad], clean[~bad]) and torch.equal(lse[~bad], clean_lse[~bad])
    p.done()


def test_keys_of_nan_over_whole_runs_give_nan():
    """Behind every number of blocks of 64 keys, wherever the runs end: what sees NaN is NaN."""
    p = nan_problem([4000], [1], 4, 2, 128)
    _, clean_lse = p.run()
    for block in range(62, 0, -1):
        p.k[0][64 * block:, 1] = math.nan
        out, lse = p.run()
        assert bool(torch.isnan(out[:, 2:]).all()) and bool(torch.isnan(lse[:, 2:]).all()), block
        assert torch.equal(lse[:, :2], clean_lse[:, :2])
    p.done()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("new,d", [(1, 64), (40, 128), (100, 64), (100, 256)])
def test_an_infinite_value_of_a_small_weight(dtype, new, d):
    """exp(-60) of the largest weight is no number of fp16, but it is not zero: infinite values give infinities, one part of the weights or several."""
    p = Problem(91, [700], [new], 4, 1, d, dtype, dtype, tree=[random_tree(new, 7)])
    p.scale = 0.125
    p.q.view(new, 4, d)[..., 0] = 8.0
    p.k[0][:, 0, 0] = 0.0
    p.k[0][[20, 300], 0, 0] = -60.0
    p.v[0][20, 0, 5], p.v[0][300, 0, 9] = math.inf, -math.inf
    out, lse = p.run()
    assert bool((out[..., 5] == math.inf).all()) and bool((out[..., 9] == -math.inf).all())
    assert int((~torch.isfinite(out)).sum()) == 2 * new * 4 and bool(torch.isfinite(lse).all())
    p.done()


@pytest.mark.parametrize("new,out", [(10, "bf16"), (20, "f32"), (20, "bf16")])
def test_many_sequences_of_many_rows(new, out):
    """More than a wave looks at in one go, through tiles of 64 and of 128 rows; some have no tokens."""
    g = torch.Generator()
    g.manual_seed(9)
    ctx = torch.randint(0, 150, (140,), generator=g).tolist()
    p = Problem(101, ctx, [0 if i % 13 == 4 else new + i % 3 for i in range(140)], 4, 1, 64, "bf16", out)
    got, lse = p.run()
    p.check(got, lse)
    p.done()


@pytest.mark.parametrize("dtype,out", [("f16", "f16"), ("f16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("new,cap", [(1, 0.0), (10, 0.0), (60, 0.0), (60, 15.0)])
def test_negative_scales(dtype, out, new, cap):
    """Minus the scale is minus the queries (not to the bit: sums of the matrix instructions are not rounded alike for both signs)."""
    p = Problem(111, [300], [new], 4, 1, 64, dtype, out, cap=cap)
    p.scale, p.q = -p.scale, -p.q
    got, lse = p.run()
    p.scale, p.q = -p.scale, -p.q
    p.check(got, lse)
    p.done()
