"""The example's trees of drafted tokens, of any size: rows packed in words (no GPU needed), and tokens that do not depend on them."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("nodes", [1, 31, 32, 33, 70])
def test_rows_of_any_length_are_packed(nodes):
    import draft_decode
    rows = [(1 << j) | 1 for j in range(nodes)]
    words = draft_decode.Server._pack(rows, nodes).numpy().view(np.uint32)
    assert words.shape == (nodes, -(-nodes // 32))
    for j in range(nodes):
        assert [i for i in range(32 * words.shape[1]) if words[j, i // 32] >> (i % 32) & 1] == sorted({0, j})


@pytest.mark.gpu
def test_many_drafts_do_not_change_the_tokens():
    import draft_decode
    model = draft_decode.Model(vocab=60)
    prompt = [int(t) for t in np.random.default_rng(8).integers(0, 6, 60)]
    many, few = (draft_decode.generate(model, prompt, 30, greedy=True, drafts=d) for d in (40, 0))
    model.close()
    assert many[:2] == few[:2]


@pytest.mark.gpu
def test_a_prompt_of_one_token():
    import draft_decode
    model = draft_decode.Model(vocab=60)
    many, few = (draft_decode.generate(model, [7], 12, greedy=True, drafts=d) for d in (5, 0))
    model.close()
    assert many[:2] == few[:2] and len(few[0]) == 12


def test_a_fork_drafts_from_its_own_tokens():
    from types import SimpleNamespace

    import draft_decode
    seq = {"pages": [0], "length": 16, "tokens": list(range(17)), "follows": {3: [4]}}
    other = draft_decode.Server.fork(SimpleNamespace(users=[1], page=16), seq)
    other["follows"][3].append(9)
    other["pages"].append(1)
    other["tokens"].append(5)
    assert seq["follows"] == {3: [4]} and seq["pages"] == [0] and len(seq["tokens"]) == 17
