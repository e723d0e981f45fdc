"""Workspaces that serve smaller calls as well: a program that asks once, for the largest batch it will have, is not refused later (no GPU needed)."""
import random

import pytest

from paper_2602_06694_amd import binding as nq

HEADS = [(64, 8, 128), (32, 32, 128), (8, 1, 64), (28, 4, 256), (6, 3, 80)]


def attention(hq, hk, d):
    kv = nq.nq_kv_create(1 << 20, 1 << 20, nq.NQ_BF16, hk, d, 16, 8)
    a = nq.nq_attn_create(kv, hq, 1.0, 0.0, nq.NQ_BF16)
    nq.nq_kv_destroy(kv)
    return a


@pytest.mark.parametrize("hq,hk,d", HEADS)
def test_attention_of_smaller_batches(hq, hk, d):
    a = attention(hq, hk, d)
    room = lambda s, t: nq.nq_attn_workspace_bytes(a, s, t)  # noqa: E731
    assert room(1, 64) <= room(32, 64) <= room(32, 65)
    r = random.Random(1)
    for _ in range(3000):
        seqs, tokens = int(2 ** r.uniform(0, 9)), int(2 ** r.uniform(0, 12))
        fewer = r.randint(1, seqs), r.randint(0, tokens)
        assert room(*fewer) <= room(seqs, tokens), (fewer, seqs, tokens)
    # what a call itself needs by its cut: items of a key head times the rows of a tile, 4 floats beside each row's elements
    group, wide = hq // hk, 64 if d <= 64 else 128 if d <= 128 else 256
    for seqs, tokens in ((1, 1), (32, 32), (32, 64), (1, 64), (1, 2048), (5, 90), (256, 256)):
        mean = max(1, tokens * group // seqs)
        rows = 16 if mean <= 16 else 64 if mean <= 64 or wide == 256 else 128
        slots = max(1, (1 if wide == 256 and rows == 16 else 2) * 256 // hk)
        assert room(seqs, tokens) >= (2 * slots + tokens * group // rows + seqs) * hk * rows * (wide + 4) * 4
    nq.nq_attn_destroy(a)


def test_sampling_of_fewer_rows():
    room = nq.nq_sample_workspace_bytes
    part = 8 * 2048 + 4 * 2048 + 16                         # a part's sums, counts and the rest
    parts = lambda n, vocab: max(1, min(-(-768 // n), vocab // 16384, 8)) * n  # noqa: E731
    for vocab in (1000, 16384, 32000, 32768, 60000, 131071, 262144, 1 << 20):
        sizes = [room(n, vocab) for n in range(0, 1700)]
        assert sizes == sorted(sizes), vocab
        for n in range(1, 1700):
            assert sizes[n] >= (parts(n, vocab) * part if parts(n, vocab) > n else 0)
        assert sizes[-1] <= room(1699, 1 << 20)
    r = random.Random(2)
    for _ in range(2000):
        n, vocab = int(2 ** r.uniform(0, 13)), int(2 ** r.uniform(0, 20))
        assert room(r.randint(0, n), r.randint(1, vocab)) <= room(n, vocab)
