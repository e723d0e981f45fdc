"""How attention's work is numbered, in a model of the kernels' arithmetic (no GPU needed): every item of a list that rises is found once and has its place, and what lists of any
other order leave stays within the workspace."""
import random

import numpy as np
import pytest

from paper_2602_06694_amd import binding as nq

NO_RUNS, BLOCK, MIN_RUN = 1 << 25, 64, 2
f32 = np.float32


class Call:
    def __init__(self, begin, ctx, n_tokens, hq, hk, table=1 << 20, page=16, cus=256, dim=128):
        self.n_tokens, self.group, self.n_seqs = n_tokens, hq // hk, len(ctx)
        mean = max(1, n_tokens * self.group // self.n_seqs)
        self.rows = 16 if mean <= 16 else 64 if mean <= 64 or dim > 128 else 128
        self.slots = max(1, (1 if dim > 128 and self.rows == 16 else 2) * cus // hk)
        self.items = 2 * self.slots + n_tokens * self.group // self.rows + self.n_seqs
        self.tiles, self.blocks = [], []
        for s, c in enumerate(ctx):
            first = min(max(begin[s], 0), n_tokens)
            n = min(max(begin[s + 1], first), n_tokens) - first
            keys = min(max(c, 0) + n, min(table * page, 2 ** 31 - 1 - 4096))
            self.tiles.append(-(-n * self.group // self.rows))
            self.blocks.append(-(-keys // BLOCK) if n else 0)
        self.run = self.run_length()

    def run_length(self):
        """Blocks of a run; divisions in fp32, as on the device."""
        over = lambda x, y: int(min(f32(x) * (f32(1.0000002) / f32(y)), f32(NO_RUNS))) + 1  # noqa: E731
        work, tiles, longest = sum(t * b for t, b in zip(self.tiles, self.blocks)), max(1, sum(self.tiles)), max(self.blocks)
        blocks, cost = f32(work), 2.0 if self.rows == 16 else 4.0
        rounds, places = -(-tiles // self.slots), self.slots // tiles
        whole = max(f32(longest), blocks * f32(rounds) / f32(tiles))
        fit = NO_RUNS if places == 0 else min(-(-longest // places), NO_RUNS if places == 1 else over(blocks, f32(self.slots) - f32(tiles)) if self.slots > tiles else NO_RUNS)
        half = over(blocks, 2 * self.slots)
        at_once, in_turn = fit + cost + 3, 2.5 * half + 2 * cost + 3
        if whole <= min(at_once, in_turn):
            return NO_RUNS
        return max(MIN_RUN, fit if at_once <= in_turn else half)

    def runs(self, s):
        return -(-self.blocks[s] // self.run)

    def item(self, number, bounded=True):
        """(sequence, tile, run, place or None) or None."""
        before = 0
        for s in range(self.n_seqs):
            count = min(self.tiles[s] * self.runs(s), self.items + 1)
            if before + count > number:
                if bounded and self.runs(s) > 1 and before + count > self.items:
                    return None
                run, at = divmod(number - before, self.tiles[s])
                tile = self.tiles[s] - 1 - at
                return s, tile, run, before + tile + run * self.tiles[s] if self.runs(s) > 1 else None
            before += count
        return None

    def found(self, bounded=True):
        return [i for i in (self.item(n, bounded) for n in range(self.items)) if i]


FALLING = [([0, 2048] * 5, [30000] * 9, 2048, 8, 8), ([0, 320] * 7, [64] * 12 + [60000], 320, 64, 8)]


@pytest.mark.parametrize("begin,ctx,n_tokens,hq,hk", FALLING)
def test_lists_that_do_not_rise_stay_within_the_workspace(begin, ctx, n_tokens, hq, hk):
    call = Call(begin[:len(ctx) + 1], ctx, n_tokens, hq, hk)
    places = lambda bounded: [p for _, _, _, p in call.found(bounded) if p is not None]  # noqa: E731
    assert max(places(False)) >= call.items             # (these lists do ask for more than there is)
    assert all(p < call.items for p in places(True))


@pytest.mark.parametrize("seed", range(200))
def test_any_list(seed):
    r = random.Random(seed)
    hq, hk = r.choice([(32, 32), (64, 8), (8, 1), (28, 4), (1, 1)])
    n_seqs = r.choice([1, 2, 5, 63, 64, 65, 130])
    n_tokens = r.choice([1, 7, n_seqs, 3 * n_seqs, 300, 2048])
    ctx = [int(2 ** r.uniform(-1, 18)) for _ in range(n_seqs)]
    if r.random() < 0.5:                                # any numbers
        begin = [r.randint(-5, n_tokens + 5) for _ in range(n_seqs + 1)]
        call = Call(begin, ctx, n_tokens, hq, hk, table=r.choice([1, 3, 1 << 20]))
        assert all(p is None or p < call.items for _, _, _, p in call.found())
        return
    begin = [0] + sorted(r.randint(0, n_tokens) for _ in range(n_seqs - 1)) + [n_tokens]
    call = Call(begin, ctx, n_tokens, hq, hk)
    want = {(s, t, k) for s in range(n_seqs) for t in range(call.tiles[s]) for k in range(call.runs(s))}
    found = call.found()
    assert {i[:3] for i in found} == want and len(found) == len(want)
    places = [p for _, _, _, p in found if p is not None]
    assert len(set(places)) == len(places) and all(p < call.items for p in places)


def test_calls_of_more_items_than_a_launch_has_are_refused():
    kv = nq.nq_kv_create(1 << 20, 1 << 20, nq.NQ_BF16, 2, 64, 16, 8)
    a = nq.nq_attn_create(kv, 4, 1.0, 0.0, nq.NQ_BF16)
    nq.nq_kv_destroy(kv)
    assert nq.nq_attn_workspace_bytes(a, 1 << 22, 1 << 22) > 0
    for n_seqs, n_tokens in ((1 << 23, 1 << 23), (1 << 23, 1), (1 << 28, 1)):
        with pytest.raises(nq.NQError) as e:
            nq.nq_attn_workspace_bytes(a, n_seqs, n_tokens)
        assert e.value.status == nq.NQ_E_SHAPE
    nq.nq_attn_destroy(a)
