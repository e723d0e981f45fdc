"""Rotary halves that are no whole chunks of eight, in 16-bit types (read in two pieces and turned round by every amount), and batches of tokens beyond one to a workgroup."""
import pytest
import torch

import test_gpu_rope as base
from paper_2602_06694_amd import binding as nq
from decoder_util import NQ, TORCH, Cache, close, frequencies, randn, rope

pytestmark = pytest.mark.gpu

HALVES = [(80, 34), (80, 36), (80, 38), (80, 2), (80, 78), (256, 34), (256, 36), (256, 38), (256, 42), (256, 250), (24, 22), (8, 6)]       # head_dim, rot_dim
TYPES = [("bf16", "bf16"), ("f16", "f16"), ("f16", "bf16"), ("bf16", "f16")]


@pytest.mark.parametrize("d,rot", HALVES)
@pytest.mark.parametrize("tin,tout", TYPES)
def test_forward_and_backward(d, rot, tin, tout):
    case = (7, 5, 1, d, rot, nq.NQ_ROPE_HALF, True, tin, tout)
    base.test_forward(case)
    base.test_backward(case)


@pytest.mark.parametrize("d,rot", HALVES)
@pytest.mark.parametrize("t", ["bf16", "f16"])
def test_in_place_and_into_the_cache(d, rot, t):
    n, hq, hk, page = 21, 6, 3, 16
    q, k, v = (randn(i, n, h * d).to(TORCH[t]).cuda() for i, h in ((61, hq), (62, hk), (63, hk)))
    pos = (torch.arange(n) * 7 + 3).int()
    f = frequencies(rot)
    w = (1 + 0.2 * randn(64, d)).float()
    r = nq.nq_rope_create(hq, hk, d, rot, nq.NQ_ROPE_HALF, f, 1.0, 1e-6, 0.0, NQ[t], NQ[t])
    qo, ko, qc = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q)
    nq.nq_rope_forward(r, q, k, w.cuda(), w.cuda(), pos.cuda(), qo, ko)
    cache = Cache(hk, d, page, 2, t)
    nq.nq_rope_cache(r, cache.handles[0], q, k, v, w.cuda(), w.cuda(), pos.cuda(), torch.arange(n, device="cuda"), qc)
    torch.cuda.synchronize()
    kc, vc = (cache.view(i).transpose(1, 2).reshape(2 * page, hk, d)[:n] for i in (0, 1))
    for x, heads, got in ((q, hq, qo.view(n, hq, d)), (q, hq, qc.view(n, hq, d)), (k, hk, ko.view(n, hk, d)), (k, hk, kc)):
        x = x.double().cpu().view(n, heads, d)
        close(got, rope(x, w, pos.numpy(), f, rot, nq.NQ_ROPE_HALF, 1e-6), t, base.slack(x, w, rot, nq.NQ_ROPE_HALF, 1e-6, 0.0, 1.0))
    assert torch.equal(vc.reshape(n, hk * d), v)
    dq, dk = randn(65, n, hq * d).to(TORCH[t]).cuda(), randn(66, n, hk * d).to(TORCH[t]).cuda()
    room = torch.empty(nq.nq_rope_backward_workspace_bytes(r, n), dtype=torch.uint8, device="cuda")
    apart = [torch.empty_like(dq), torch.empty_like(dk), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")]
    within = [dq.clone(), dk.clone(), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")]
    nq.nq_rope_backward(r, q, k, w.cuda(), w.cuda(), pos.cuda(), dq, dk, *apart, room, room.numel())
    nq.nq_rope_backward(r, q, k, w.cuda(), w.cuda(), pos.cuda(), within[0], within[1], *within, room, room.numel())
    nq.nq_rope_forward(r, q, k, w.cuda(), w.cuda(), pos.cuda(), q, k)
    torch.cuda.synchronize()
    nq.nq_rope_destroy(r)
    cache.close()
    assert torch.equal(q, qo) and torch.equal(k, ko)
    assert all(torch.equal(a, b) for a, b in zip(apart, within))


@pytest.mark.parametrize("case", [
    (4500, 2, 1, 8, 8, nq.NQ_ROPE_HALF, True, "bf16", "bf16"), (9001, 2, 1, 8, 6, nq.NQ_ROPE_HALF, True, "f16", "f16"), (9001, 2, 2, 16, 16, nq.NQ_ROPE_INTERLEAVED, False, "bf16", "bf16"),
    (9001, 1, 1, 256, 256, nq.NQ_ROPE_HALF, True, "f32", "bf16"),       # four tokens' angles at a time, the backward's workgroups have nine
])
def test_several_tokens_to_a_workgroup(case):
    base.test_forward(case)
    base.test_backward(case)
